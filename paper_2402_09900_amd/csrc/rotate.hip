// rotate.hip -- queries and keys of a layer: RMS norm per head and the rotation
// by position, in one pass, and its gradient.
//
// Per row x of d elements (one head of one step), with r = rsqrt(mean x^2 + eps),
//     y = x r w  (y = x without a weight),   pair p of y turned by angle
//     position freq_p, p < rot / 2, the rest of the row as it is.
// Gradient, with gy the upstream gradient turned back:
//     dw = sum over rows of gy x r,   dx = r gy w - x r^3 mean(gy w x).
//
// Bound by memory: every element read once and written once (gradient: x and the
// upstream gradient read), 10 (gradient: 30) flops each.  65536 steps of 16 + 16
// heads of 128, bf16: 192 us, 5.6 TB/s.  32768 steps of 32 + 8 heads of 128, bf16: 123
// us forward, gradient 206 (4.9 TB/s) and 6 for the weights' sums; 32768 steps of 16 +
// 16 heads of 128, fp32: a call of either 205 and 312 us, 5.2 TB/s.
//
// A lane holds two runs of CH elements, A and B, that are the halves of its CH pairs
// (half layout: elements p and p + rot / 2; interleaved: the even and odd ones of
// 2 CH in a row), so a pair never crosses lanes; LPR lanes hold a row and a wavefront
// the rows of one step of q or of k, several at a time.  Wavefronts with rows of both
// held two sets of weights and of their sums: two of them on a SIMD instead of three,
// and 279 us for the gradient above.  The angles of a step are formed once for all
// its rows, a pair per lane, while the rows are on their way, and handed on through
// LDS: in 64 bits down to the fraction of a turn (position 1e5 times frequency 1 has
// 7 bits left behind the point in 32), then sine and cosine in 32.
#include "scan_common.hpp"
#include "kernels.hpp"

namespace memoroid {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kPairs = kRotMaxDim / 2;
static_assert(kPairs == 64, "a lane per pair");

// CH elements as they lie in memory
template <int BF16, int CH>
struct Raw {
    static constexpr int WORDS = BF16 ? (CH + 1) / 2 : CH;
    uint32_t w[WORDS];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int e = 0; e < WORDS; ++e) w[e] = 0u;
    }
    __device__ __forceinline__ void load(const void* p, int64_t i) {
        if constexpr (BF16 && CH == 1) {
            w[0] = ((const uint16_t*)p)[i];
        } else {
            const uint32_t* const s = (const uint32_t*)((const char*)p + i * (BF16 ? 2 : 4));
            if constexpr (WORDS == 4) *(u32x4*)w = *(const u32x4*)s;
            else if constexpr (WORDS == 2) *(u32x2*)w = *(const u32x2*)s;
            else w[0] = *s;
        }
    }
    __device__ __forceinline__ void values(float (&v)[CH]) const {
#pragma unroll
        for (int e = 0; e < CH; ++e) {
            if constexpr (BF16) v[e] = e & 1 ? bf16_hi(w[e / 2]) : __uint_as_float(w[e / 2] << 16);
            else v[e] = __uint_as_float(w[e]);
        }
    }
};
template <int BF16, int CH>
__device__ __forceinline__ void store_run(const float (&v)[CH], void* p, int64_t i) {
    if constexpr (BF16 && CH == 1) {
        ((uint16_t*)p)[i] = (uint16_t)f32_to_bf16(v[0]);
    } else {
        uint32_t w[Raw<BF16, CH>::WORDS];
#pragma unroll
        for (int e = 0; e < Raw<BF16, CH>::WORDS; ++e) {
            if constexpr (BF16) w[e] = f32x2_to_bf16x2(v[2 * e], v[2 * e + 1]);
            else w[e] = __float_as_uint(v[e]);
        }
        uint32_t* const s = (uint32_t*)((char*)p + i * (BF16 ? 2 : 4));
        if constexpr (Raw<BF16, CH>::WORDS == 4) *(u32x4*)s = *(u32x4*)w;
        else if constexpr (Raw<BF16, CH>::WORDS == 2) *(u32x2*)s = *(u32x2*)w;
        else *s = w[0];
    }
}

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

// cosine and sine of this lane's pair of a step, times the amplitude (of a pair that
// is turned).  turns: of the pair, per position
__device__ __forceinline__ void angle(float (&cs)[2], double turns, int32_t position, float amplitude) {
    const double x = (double)position * turns;
    float s, c;
    sincospif(2.0f * (float)(x - rint(x)), &s, &c);
    cs[0] = c * amplitude;
    cs[1] = s * amplitude;
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
    __shared__ double sDw[GRAD ? 4 : 1][GRAD ? kRotMaxDim : 1];
    __shared__ double sSum[GRAD ? 2 * CH : 1][GRAD ? 256 : 1];   // a lane's sums past 64 rows
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (p.hdr && blockIdx.x == 0 && threadIdx.x < 16) {
        const u32x4 ones = {kEmpty32, kEmpty32, kEmpty32, kEmpty32};
        const u32x4 head = {kEmpty32, kEmpty32, (uint32_t)p.sig, (uint32_t)(p.sig >> 32)};
        ((u32x4*)p.hdr)[threadIdx.x] = threadIdx.x == 0 ? head : ones;
    }
    // a workgroup has rows of q or rows of k: one set of weights and of their sums
    const bool keys = (int)blockIdx.x >= p.side[0].groups;
    const RotateSide& S = p.side[keys ? 1 : 0];
    const int group = (int)blockIdx.x - (keys ? p.side[0].groups : 0);
    const int lpr = p.lpr, rpw = 64 / lpr;
    const int sub = lane / lpr;
    const RotLane<CH> L(lane % lpr, p.d, p.rot, p.inter);
    const int per = (S.H + S.parts - 1) / S.parts;
    const float inv_d = 1.0f / (float)p.d;
    const bool norm = S.w != nullptr;
    // the lane's weights, in pairs
    float wa[CH], wb[CH], da[CH], db[CH];
#pragma unroll
    for (int e = 0; e < CH; ++e) {
        wa[e] = norm && L.in ? S.w[L.first + e] : 1.0f;
        wb[e] = norm && L.in ? S.w[L.second + e] : 1.0f;
        da[e] = db[e] = 0.0f;
    }
    to_pairs<CH>(wa, wb, p.inter);
    // Sums of the weights' gradients are in floats over 64 rows, then in doubles: a
    // lane's rows grow with the call, and floats would add up their roundings.
    if constexpr (GRAD) {
#pragma unroll
        for (int e = 0; e < 2 * CH; ++e) sSum[e][threadIdx.x] = 0.0;
    }
    auto put_by = [&] {
        if constexpr (GRAD) {
#pragma unroll
            for (int e = 0; e < CH; ++e) {
                sSum[e][threadIdx.x] += (double)da[e];
                sSum[CH + e][threadIdx.x] += (double)db[e];
                da[e] = db[e] = 0.0f;
            }
        }
    };
    int rows = 0;                                          // in da, db
    // whether the lane's pair e is turned: a selection, since a factor of 0 would make
    // its neighbour's infinity a NaN
    const int turned_pairs = p.rot / 2 - L.pair0;
    auto turned = [&](int e) { return e < turned_pairs; };
    const double turns = lane < p.rot / 2 ? (double)p.freq[lane] * 0.15915494309189533577 : 0.0;   // 1 / 2 pi
    constexpr int NR = 2;                                  // rows of a lane in flight
    Raw<BF16, CH> xa[NR], xb[NR], ya[GRAD ? NR : 1], yb[GRAD ? NR : 1];
    auto fetch = [&](int64_t at0, int row0, int r1) {
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int row = row0 + i * rpw;
            const bool in = L.in && row < r1;
            const int64_t at = at0 + (int64_t)row * p.d;
            xa[i].zero();
            xb[i].zero();
            if (in && (!GRAD || norm)) {                   // (a gradient without a norm does not need x)
                xa[i].load(S.x, at + L.first);
                xb[i].load(S.x, at + L.second);
            }
            if constexpr (GRAD) {
                ya[i].zero();
                yb[i].zero();
                if (in) {
                    ya[i].load(S.g, at + L.first);
                    yb[i].load(S.g, at + L.second);
                }
            }
        }
    };
    const int64_t waves = (int64_t)S.groups * 4, tasks = p.n * S.parts;
    for (int64_t task = (int64_t)group * 4 + w; task < tasks; task += waves) {
        const int64_t t = task / S.parts, at0 = t * S.H * p.d;
        const int r0 = (int)(task % S.parts) * per, r1 = r0 + per < S.H ? r0 + per : S.H;
        const int32_t position = p.rot ? p.positions[t] : 0;
        fetch(at0, r0 + sub, r1);                          // before the angles
        wave_lds_fence();                                  // the last step's angles have been read
        angle(sCs[w][lane], turns, position, p.amplitude);
        wave_lds_fence();
        float c[CH], s[CH];
#pragma unroll
        for (int e = 0; e < CH; ++e) {
            c[e] = L.in ? sCs[w][L.pair0 + e][0] : 1.0f;
            s[e] = L.in ? sCs[w][L.pair0 + e][1] : 0.0f;
        }
        for (int row0 = r0 + sub; row0 - sub < r1; row0 += NR * rpw) {
            if (row0 != r0 + sub) fetch(at0, row0, r1);
            if (GRAD && rows >= 64) {
                put_by();
                rows = 0;
            }
            rows += NR;
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                if (row0 - sub + i * rpw >= r1) break;     // no lane has a row
                const int row = row0 + i * rpw;
                const bool in = L.in && row < r1;
                const int64_t at = at0 + (int64_t)row * p.d;
                float a[CH], b[CH], r = 1.0f;
                if (!GRAD || norm) {
                    xa[i].values(a);
                    xb[i].values(b);
                    to_pairs<CH>(a, b, p.inter);
                }
                if (norm) {
                    float sq = 0.0f;
#pragma unroll
                    for (int e = 0; e < CH; ++e) sq = __builtin_fmaf(a[e], a[e], __builtin_fmaf(b[e], b[e], sq));
                    sq = row_sum(sq, lpr);
                    // past the last row nothing is normed: eps may be 0
                    if (row < r1) r = rsqrtf(__builtin_fmaf(sq, inv_d, p.eps));
                }
                if constexpr (!GRAD) {
#pragma unroll
                    for (int e = 0; e < CH; ++e) {
                        const float x = a[e] * (r * wa[e]), y = b[e] * (r * wb[e]);
                        a[e] = turned(e) ? x * c[e] - y * s[e] : x;
                        b[e] = turned(e) ? y * c[e] + x * s[e] : y;
                    }
                    from_pairs<CH>(a, b, p.inter);
                    if (in) {
                        store_run<BF16, CH>(a, S.out, at + L.first);
                        store_run<BF16, CH>(b, S.out, at + L.second);
                    }
                } else {
                    float ga[CH], gb[CH];
                    ya[i].values(ga);
                    yb[i].values(gb);
                    to_pairs<CH>(ga, gb, p.inter);
#pragma unroll
                    for (int e = 0; e < CH; ++e) {
                        const float x = ga[e], y = gb[e];
                        ga[e] = turned(e) ? x * c[e] + y * s[e] : x;
                        gb[e] = turned(e) ? y * c[e] - x * s[e] : y;
                    }
                    if (norm) {
                        float dot = 0.0f;
#pragma unroll
                        for (int e = 0; e < CH; ++e) {
                            da[e] = __builtin_fmaf(ga[e] * a[e], r, da[e]);
                            db[e] = __builtin_fmaf(gb[e] * b[e], r, db[e]);
                            ga[e] *= wa[e];
                            gb[e] *= wb[e];
                            dot = __builtin_fmaf(ga[e], a[e], __builtin_fmaf(gb[e], b[e], dot));
                        }
                        dot = row_sum(dot, lpr);
                        const float f = dot * inv_d * r * r * r;
#pragma unroll
                        for (int e = 0; e < CH; ++e) {
                            ga[e] = __builtin_fmaf(-f, a[e], r * ga[e]);
                            gb[e] = __builtin_fmaf(-f, b[e], r * gb[e]);
                        }
                    }
                    from_pairs<CH>(ga, gb, p.inter);
                    if (in) {
                        store_run<BF16, CH>(ga, S.out, at + L.first);
                        store_run<BF16, CH>(gb, S.out, at + L.second);
                    }
                }
            }
        }
    }
    if constexpr (GRAD) {
        if (!p.part) return;
        // the lanes of a column, then the four wavefronts, in a fixed order
        put_by();
        double a[CH], b[CH];
#pragma unroll
        for (int e = 0; e < CH; ++e) {
            a[e] = sSum[e][threadIdx.x];
            b[e] = sSum[CH + e][threadIdx.x];
#pragma unroll
            for (int m = 1; m < 64; m <<= 1)
                if (m >= lpr) {
                    a[e] += __shfl_xor(a[e], m, 64);
                    b[e] += __shfl_xor(b[e], m, 64);
                }
        }
        if (sub == 0 && L.in)
#pragma unroll
            for (int e = 0; e < CH; ++e) {
                // pairs as they lie in memory: halves, or one behind the other
                sDw[w][p.inter ? L.first + 2 * e : L.first + e] = a[e];
                sDw[w][p.inter ? L.first + 2 * e + 1 : L.second + e] = b[e];
            }
        __syncthreads();
        for (int i = threadIdx.x; i < p.d; i += 256)
            p.part[(int64_t)blockIdx.x * p.d + i] =
                (float)((sDw[0][i] + sDw[GRAD ? 1 : 0][i]) + (sDw[GRAD ? 2 : 0][i] + sDw[GRAD ? 3 : 0][i]));
    }
}

// dwq = sum of part[0 .. qgroups - 1][d], dwk = of the groups behind, in 64 bits: 16
// columns per workgroup, 256 rows of 4 of them at a time, all in flight (2048 groups of
// 128: 4 us, 8 with 64 rows at a time)
__global__ __launch_bounds__(1024) void rotate_weights_kernel(const float* part, float* dwq, float* dwk, int qgroups,
                                                              int groups, int d) {
    __shared__ double sSum[16][16];
    const int unit = threadIdx.x & 3, row = threadIdx.x >> 2, col = (int)blockIdx.x * 16 + unit * 4;
    float* const out = blockIdx.y ? dwk : dwq;
    if (!out) return;
    const int i0 = blockIdx.y ? qgroups : 0, i1 = blockIdx.y ? groups : qgroups;
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (int base = i0; base < i1; base += 256 * 8) {
        f32x4 x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int i = base + 256 * k + row;
            x[k] = i < i1 && col < d ? *(const f32x4*)(part + (int64_t)i * d + col) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += (double)x[k][e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (int m = 4; m < 64; m <<= 1) s[e] += __shfl_xor(s[e], m, 64);
        if ((threadIdx.x & 63) < 4) sSum[threadIdx.x >> 6][unit * 4 + e] = s[e];
    }
    __syncthreads();
    const int i = threadIdx.x, at = (int)blockIdx.x * 16 + i;
    if (i < 16 && at < d) {
        double sum = 0.0;
        for (int k = 0; k < 16; ++k) sum += sSum[k][i];
        out[at] = (float)sum;
    }
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

hipError_t rotate_launch(bool bf16, bool grad, int ch, const RotateArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)(a.side[0].groups + a.side[1].groups));
    if (bf16) {
        if (grad) rotate_dispatch<1, true>(ch, grid, a, s);
        else rotate_dispatch<1, false>(ch, grid, a, s);
    } else {
        if (grad) rotate_dispatch<0, true>(ch, grid, a, s);
        else rotate_dispatch<0, false>(ch, grid, a, s);
    }
    return hipGetLastError();
}

hipError_t rotate_weights_launch(const RotateArgs& a, float* dwq, float* dwk, hipStream_t s) {
    hipLaunchKernelGGL(rotate_weights_kernel, dim3((unsigned)((a.d + 15) / 16), 2), dim3(1024), 0, s, a.part, dwq, dwk,
                       a.side[0].groups, a.side[0].groups + a.side[1].groups, a.d);
    return hipGetLastError();
}

}  // namespace memoroid
