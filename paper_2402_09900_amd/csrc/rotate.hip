// rotate.hip -- queries and keys of a layer: RMS norm per head and the rotation
// by position, in one pass, and its gradient.
//
// Per row x of d elements (one head of one step), with r = rsqrt(mean x^2 + eps),
//     y = x r w  (y = x without a weight),   pair p of y turned by angle
//     position freq_p, p < rot / 2, the rest of the row as it is.
// Gradient, with gy the upstream gradient turned back:
//     dw = sum over rows of gy x r,   dx = r gy w - x r^3 mean(gy w x).
//
// Bound by memory: every element read once and written once, 10 (gradient: 30)
// flops each.  A lane holds two runs of CH elements, A and B, that are the halves
// of its CH pairs (half layout: elements p and p + rot / 2; interleaved: the even
// and odd ones of 2 CH in a row), so a pair never crosses lanes; LPR lanes hold a
// row and a wavefront the rows of one step, several at a time.  The angles of a
// step are formed once for all its rows, a pair per lane, and handed on through
// LDS: in 64 bits down to the fraction of a turn (position 1e5 times frequency 1
// has 7 bits left behind the point in 32), then sine and cosine in 32.
#include "scan_common.hpp"
#include "kernels.hpp"

namespace memoroid {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kPairs = kRotMaxDim / 2;

template <int BF16, int CH>
struct Run {
    float v[CH];
    __device__ __forceinline__ void load(const void* p, int64_t i) {
        if constexpr (BF16) {
            const uint16_t* const s = (const uint16_t*)p + i;
            uint32_t w[(CH + 1) / 2];
            if constexpr (CH == 8) *(u32x4*)w = *(const u32x4*)s;
            else if constexpr (CH == 4) *(u32x2*)w = *(const u32x2*)s;
            else if constexpr (CH == 2) w[0] = *(const uint32_t*)s;
            else w[0] = *s;
#pragma unroll
            for (int e = 0; e < CH; ++e) v[e] = e & 1 ? bf16_hi(w[e / 2]) : __uint_as_float(w[e / 2] << 16);
        } else {
            const float* const s = (const float*)p + i;
            if constexpr (CH == 4) *(f32x4*)v = *(const f32x4*)s;
            else
#pragma unroll
                for (int e = 0; e < CH; ++e) v[e] = s[e];
        }
    }
    __device__ __forceinline__ void store(void* p, int64_t i) const {
        if constexpr (BF16) {
            uint16_t* const s = (uint16_t*)p + i;
            if constexpr (CH == 1) {
                *s = (uint16_t)f32_to_bf16(v[0]);
            } else {
                uint32_t w[CH / 2];
#pragma unroll
                for (int e = 0; e < CH / 2; ++e) w[e] = f32x2_to_bf16x2(v[2 * e], v[2 * e + 1]);
                if constexpr (CH == 8) *(u32x4*)s = *(u32x4*)w;
                else if constexpr (CH == 4) *(u32x2*)s = *(u32x2*)w;
                else *(uint32_t*)s = w[0];
            }
        } else {
            float* const s = (float*)p + i;
            if constexpr (CH == 4) *(f32x4*)s = *(const f32x4*)v;
            else
#pragma unroll
                for (int e = 0; e < CH; ++e) s[e] = v[e];
        }
    }
};

// A lane's place in a row: where its runs lie, and its pairs
template <int CH>
struct RotLane {
    int first, second, pair0;
    bool in;
    __device__ RotLane(int unit, int d, int rot, bool inter) {
        in = unit * 2 * CH < d;
        pair0 = unit * CH;
        // half layout: the pairs, then the rest in runs one behind the other
        const bool turned = !inter && pair0 < rot / 2;
        first = turned ? pair0 : 2 * pair0;
        second = turned ? pair0 + rot / 2 : 2 * pair0 + CH;
    }
};
// memory order (runs) <-> pairs: interleaved runs hold A and B in turn
template <int CH>
__device__ __forceinline__ void to_pairs(float (&a)[CH], float (&b)[CH], bool inter) {
    if (!inter) return;
    float m[2 * CH];
#pragma unroll
    for (int e = 0; e < CH; ++e) {
        m[e] = a[e];
        m[CH + e] = b[e];
    }
#pragma unroll
    for (int e = 0; e < CH; ++e) {
        a[e] = m[2 * e];
        b[e] = m[2 * e + 1];
    }
}
template <int CH>
__device__ __forceinline__ void from_pairs(float (&a)[CH], float (&b)[CH], bool inter) {
    if (!inter) return;
    float m[2 * CH];
#pragma unroll
    for (int e = 0; e < CH; ++e) {
        m[2 * e] = a[e];
        m[2 * e + 1] = b[e];
    }
#pragma unroll
    for (int e = 0; e < CH; ++e) {
        a[e] = m[e];
        b[e] = m[CH + e];
    }
}

// cosine and sine of every pair of a step, times the amplitude; (1, 0) for the
// pairs that are not turned
__device__ __forceinline__ void angles(float (*cs)[2], int pairs, const float* freq, int rot, int32_t position,
                                       float amplitude, int lane) {
    for (int p = lane; p < pairs; p += 64) {
        float c = 1.0f, s = 0.0f;
        if (p < rot / 2) {
            const double turns = (double)position * (double)freq[p] * 0.15915494309189533577;   // 1 / 2 pi
            sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
            c *= amplitude;
            s *= amplitude;
        }
        cs[p][0] = c;
        cs[p][1] = s;
    }
}
// sum over the lanes of a row
__device__ __forceinline__ float row_sum(float v, int lpr) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1)
        if (m < lpr) v += lanes_xor(v, m);
    return v;
}
__device__ __forceinline__ void wave_lds_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <int BF16, int CH, bool GRAD>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs p) {
    __shared__ float sCs[4][kPairs][2];
    __shared__ float sDw[GRAD ? 4 : 1][GRAD ? 2 * kRotMaxDim : 1];
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (p.hdr && blockIdx.x == 0 && threadIdx.x < 16) {
        const u32x4 ones = {kEmpty32, kEmpty32, kEmpty32, kEmpty32};
        const u32x4 head = {kEmpty32, kEmpty32, (uint32_t)p.sig, (uint32_t)(p.sig >> 32)};
        ((u32x4*)p.hdr)[threadIdx.x] = threadIdx.x == 0 ? head : ones;
    }
    const int lpr = p.lpr, rpw = 64 / lpr;
    const int sub = lane / lpr;
    const RotLane<CH> L(lane % lpr, p.d, p.rot, p.inter);
    const int rows = p.H + p.Hk, per = (rows + p.parts - 1) / p.parts;
    const float inv_d = 1.0f / (float)p.d;
    // the lane's weights, in pairs
    float wa[2][CH], wb[2][CH], da[2][CH], db[2][CH];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float* const wt = i ? p.wk : p.wq;
#pragma unroll
        for (int e = 0; e < CH; ++e) {
            wa[i][e] = wt && L.in ? wt[L.first + e] : 1.0f;
            wb[i][e] = wt && L.in ? wt[L.second + e] : 1.0f;
            da[i][e] = db[i][e] = 0.0f;
        }
        to_pairs<CH>(wa[i], wb[i], p.inter);
    }
    const int64_t waves = (int64_t)gridDim.x * 4, tasks = p.n * p.parts;
    for (int64_t task = (int64_t)blockIdx.x * 4 + w; task < tasks; task += waves) {
        const int64_t t = task / p.parts;
        const int r0 = (int)(task % p.parts) * per, r1 = r0 + per < rows ? r0 + per : rows;
        wave_lds_fence();                                  // the last step's angles have been read
        angles(sCs[w], p.d / 2, p.freq, p.rot, p.rot ? p.positions[t] : 0, p.amplitude, lane);
        wave_lds_fence();
        float c[CH], s[CH];
#pragma unroll
        for (int e = 0; e < CH; ++e) {
            c[e] = L.in ? sCs[w][L.pair0 + e][0] : 1.0f;
            s[e] = L.in ? sCs[w][L.pair0 + e][1] : 0.0f;
        }
        constexpr int NR = GRAD ? 2 : 4;                   // rows of a lane in flight
        for (int row0 = r0 + sub; row0 - sub < r1; row0 += NR * rpw) {
            Run<BF16, CH> a[NR], b[NR], ga[GRAD ? NR : 1], gb[GRAD ? NR : 1];
            int64_t at[NR];
            bool in[NR], isk[NR];
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                const int row = row0 + i * rpw;
                in[i] = L.in && row < r1;
                isk[i] = row >= p.H;
                at[i] = isk[i] ? (t * p.Hk + (row - p.H)) * p.d : (t * p.H + row) * p.d;
#pragma unroll
                for (int e = 0; e < CH; ++e) a[i].v[e] = b[i].v[e] = 0.0f;
                // (a gradient without a norm does not need x)
                if (in[i] && (!GRAD || (isk[i] ? p.wk : p.wq) != nullptr)) {
                    a[i].load(isk[i] ? p.k : p.q, at[i] + L.first);
                    b[i].load(isk[i] ? p.k : p.q, at[i] + L.second);
                }
                if constexpr (GRAD) {
#pragma unroll
                    for (int e = 0; e < CH; ++e) ga[i].v[e] = gb[i].v[e] = 0.0f;
                    if (in[i]) {
                        ga[i].load(isk[i] ? p.gk : p.gq, at[i] + L.first);
                        gb[i].load(isk[i] ? p.gk : p.gq, at[i] + L.second);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                to_pairs<CH>(a[i].v, b[i].v, p.inter);
                // past the last row nothing is normed: eps may be 0
                const bool norm = row0 + i * rpw < r1 && (isk[i] ? p.wk : p.wq) != nullptr;
                float r = 1.0f;
                float sq = 0.0f;
#pragma unroll
                for (int e = 0; e < CH; ++e) sq = __builtin_fmaf(a[i].v[e], a[i].v[e], __builtin_fmaf(b[i].v[e], b[i].v[e], sq));
                sq = row_sum(sq, lpr);
                if (norm) r = rsqrtf(__builtin_fmaf(sq, inv_d, p.eps));
                if constexpr (!GRAD) {
#pragma unroll
                    for (int e = 0; e < CH; ++e) {
                        const float x = a[i].v[e] * (r * (isk[i] ? wa[1][e] : wa[0][e]));
                        const float y = b[i].v[e] * (r * (isk[i] ? wb[1][e] : wb[0][e]));
                        a[i].v[e] = x * c[e] - y * s[e];
                        b[i].v[e] = y * c[e] + x * s[e];
                    }
                    from_pairs<CH>(a[i].v, b[i].v, p.inter);
                    if (in[i]) {
                        a[i].store(isk[i] ? p.k_out : p.q_out, at[i] + L.first);
                        b[i].store(isk[i] ? p.k_out : p.q_out, at[i] + L.second);
                    }
                } else {
                    to_pairs<CH>(ga[i].v, gb[i].v, p.inter);
                    float dot = 0.0f;
#pragma unroll
                    for (int e = 0; e < CH; ++e) {
                        const float x = ga[i].v[e] * c[e] + gb[i].v[e] * s[e];
                        const float y = gb[i].v[e] * c[e] - ga[i].v[e] * s[e];
                        // rows of q and of k add to different sums
                        const float ax = norm ? x * a[i].v[e] * r : 0.0f, by = norm ? y * b[i].v[e] * r : 0.0f;
                        da[0][e] += isk[i] ? 0.0f : ax;
                        db[0][e] += isk[i] ? 0.0f : by;
                        da[1][e] += isk[i] ? ax : 0.0f;
                        db[1][e] += isk[i] ? by : 0.0f;
                        ga[i].v[e] = x * (isk[i] ? wa[1][e] : wa[0][e]);
                        gb[i].v[e] = y * (isk[i] ? wb[1][e] : wb[0][e]);
                        dot = __builtin_fmaf(ga[i].v[e], a[i].v[e], __builtin_fmaf(gb[i].v[e], b[i].v[e], dot));
                    }
                    dot = row_sum(dot, lpr);
                    const float f = norm ? dot * inv_d * r * r * r : 0.0f;
#pragma unroll
                    for (int e = 0; e < CH; ++e) {
                        ga[i].v[e] = norm ? __builtin_fmaf(-f, a[i].v[e], r * ga[i].v[e]) : ga[i].v[e];
                        gb[i].v[e] = norm ? __builtin_fmaf(-f, b[i].v[e], r * gb[i].v[e]) : gb[i].v[e];
                    }
                    from_pairs<CH>(ga[i].v, gb[i].v, p.inter);
                    if (in[i]) {
                        ga[i].store(isk[i] ? p.k_out : p.q_out, at[i] + L.first);
                        gb[i].store(isk[i] ? p.k_out : p.q_out, at[i] + L.second);
                    }
                }
            }
        }
    }
    if constexpr (GRAD) {
        if (!p.part) return;
        // the wavefront's rows of a step, then its four wavefronts, in a fixed order
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int e = 0; e < CH; ++e)
#pragma unroll
                for (int m = 1; m < 64; m <<= 1)
                    if (m >= lpr) {
                        da[i][e] += lanes_xor(da[i][e], m);
                        db[i][e] += lanes_xor(db[i][e], m);
                    }
            from_pairs<CH>(da[i], db[i], p.inter);
            if (sub == 0 && L.in)
#pragma unroll
                for (int e = 0; e < CH; ++e) {
                    sDw[w][i * p.d + L.first + e] = da[i][e];
                    sDw[w][i * p.d + L.second + e] = db[i][e];
                }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * p.d; i += 256)
            p.part[(int64_t)blockIdx.x * 2 * p.d + i] = (sDw[0][i] + sDw[GRAD ? 1 : 0][i]) + (sDw[GRAD ? 2 : 0][i] + sDw[GRAD ? 3 : 0][i]);
    }
}

// the workgroups' sums, in 64 bits: one column of [groups][2 d] per wavefront
__global__ __launch_bounds__(256) void rotate_weights_kernel(const float* part, float* dwq, float* dwk, int groups, int d) {
    const int col = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (col >= 2 * d) return;
    double s = 0.0;
    for (int i = lane; i < groups; i += 64) s += (double)part[(int64_t)i * 2 * d + col];
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) s += __shfl_xor(s, m, 64);
    float* const out = col < d ? dwq : dwk;
    if (lane == 0 && out) out[col < d ? col : col - d] = (float)s;
}

namespace {
template <int BF16, bool GRAD>
void rotate_dispatch(int ch, dim3 grid, const RotateArgs& a, hipStream_t s) {
    const dim3 block(256);
    switch (ch) {
        case 8:
            if constexpr (BF16) hipLaunchKernelGGL((rotate_kernel<BF16, 8, GRAD>), grid, block, 0, s, a);
            break;
        case 4: hipLaunchKernelGGL((rotate_kernel<BF16, 4, GRAD>), grid, block, 0, s, a); break;
        case 2: hipLaunchKernelGGL((rotate_kernel<BF16, 2, GRAD>), grid, block, 0, s, a); break;
        default: hipLaunchKernelGGL((rotate_kernel<BF16, 1, GRAD>), grid, block, 0, s, a); break;
    }
}
}  // namespace

hipError_t rotate_launch(bool bf16, bool grad, int ch, int64_t groups, const RotateArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)groups);
    if (bf16) {
        if (grad) rotate_dispatch<1, true>(ch, grid, a, s);
        else rotate_dispatch<1, false>(ch, grid, a, s);
    } else {
        if (grad) rotate_dispatch<0, true>(ch, grid, a, s);
        else rotate_dispatch<0, false>(ch, grid, a, s);
    }
    return hipGetLastError();
}

hipError_t rotate_weights_launch(const float* part, float* dwq, float* dwk, int64_t groups, int d, hipStream_t s) {
    hipLaunchKernelGGL(rotate_weights_kernel, dim3((unsigned)((2 * d + 3) / 4)), dim3(256), 0, s, part, dwq, dwk,
                       (int)groups, d);
    return hipGetLastError();
}

}  // namespace memoroid
