// norm.hip -- layer norm of rows, with a residual added and dropout on the way, its
// gradient, and dropout by itself.
//
// Per row of d elements,
//     s = residual + mask x / (1 - p),   y = (s - mean) rstd w + b,
//     rstd = 1 / sqrt(mean((s - mean)^2) + eps).
// Gradient, with xh = (s - mean) rstd and gw = gy w,
//     ds = gs + rstd (gw - mean(gw) - xh mean(gw xh)),   dres = ds,
//     dx = mask ds / (1 - p),   dw = sum over rows of gy xh,   db = sum of gy.
// s is summed up again from x and the residual for the gradient, in 32 bits: read
// back from a bf16 s, xh would be off by 2^-9, and dw, a 32-bit result, with it.
//
// A lane has octets (eight elements in a row), CH of them, and R rows at a time: loads of
// all of them are under way together, and wavefronts that share a row meet once a sum for
// R rows.  Rows of up to 512 elements lie in a wavefront's lanes (short ones side by side),
// longer ones in 2 to 16 wavefronts, so that a lane keeps no more than 16 elements of the
// weight and its sums in registers.
//
// Memory bounds all of it.  32768 rows of 2048 bf16, residual and dropout: forward 94 us (0.54
// GB, 5.7 TB/s), the gradient 157 (0.81 GB, 5.1 TB/s: seven octets a lane under way, half the
// workgroups of the forward's) and 5 for the weights' sums; dropout with a residual 64.5 us
// (6.2 TB/s).  fp32, 32768 x 1024: 106, 163.  Rows of 8191 137 and 203 us where rows of 8192
// take 96 and 160: their octets straddle lines.  The gradient of rows longer than 8192 keeps
// some of two octets' sums in scratch: 4096 x 16384 in 206 us.
#include <type_traits>

#include "philox.hpp"

namespace memoroid {

namespace {

// 16 bytes at an address that is a multiple of 2 or 4
typedef uint32_t Words2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t Words4 __attribute__((ext_vector_type(4), aligned(4)));

// Eight elements in memory order.  EVEN: rows are whole octets.  Otherwise `left` of them
// lie in the row, whose rows start at any element: accesses of up to 16 bytes at that
// alignment, which the hardware takes.
template <bool BF16, bool EVEN, int POL>
struct Octet {
    static constexpr int WORDS = BF16 ? 4 : 8, SIZE = BF16 ? 2 : 4;
    using Words = typename std::conditional<BF16, Words2, Words4>::type;
    uint32_t w[WORDS];
    // wide: the row has eight elements at least.  Its last octet is then loaded from where
    // eight of them end the row, and settle() moves them down to the ones that are asked for:
    // one access for every lane, and nobody waits for it before the values are due.
    __device__ __forceinline__ void load(const void* p, int64_t i, int left, bool wide) {
#pragma unroll
        for (int e = 0; e < WORDS; ++e) w[e] = 0u;
        if (left <= 0) return;
        if (EVEN || wide) {
            const char* const at = (const char*)p + (EVEN ? i : i - (8 - left)) * SIZE;
#pragma unroll
            for (int e = 0; e < WORDS; e += 4) {
                const Words* const q = (const Words*)at + e / 4;
                const Words v = POL == kStreamAll ? __builtin_nontemporal_load(q) : *q;
                w[e] = v.x;
                w[e + 1] = v.y;
                w[e + 2] = v.z;
                w[e + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (e < left) {
                    if constexpr (BF16) w[e / 2] |= (uint32_t)((const uint16_t*)p)[i + e] << (e & 1 ? 16 : 0);
                    else w[e] = ((const uint32_t*)p)[i + e];
                }
        }
    }
    __device__ __forceinline__ void settle(int left, bool wide) {
        if (EVEN || left >= 8 || left <= 0 || !wide) return;
        const int by = 8 - left;
        if constexpr (BF16) {
#pragma unroll
            for (int e = 0; e < WORDS; ++e)
                w[e] = by & 1 ? __builtin_amdgcn_alignbit(e + 1 < WORDS ? w[e + 1] : 0u, w[e], 16) : w[e];
        }
#pragma unroll
        for (int m = BF16 ? 2 : 1; m < 8; m *= 2) {
            const int words = m * SIZE / 4;
#pragma unroll
            for (int e = 0; e < WORDS; ++e) w[e] = by & m ? (e + words < WORDS ? w[e + words] : 0u) : w[e];
        }
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (BF16) v[e] = e & 1 ? bf16_hi(w[e / 2]) : bf16_lo(w[e / 2]);
            else v[e] = __uint_as_float(w[e]);
        }
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
        for (int e = 0; e < WORDS; ++e) {
            if constexpr (BF16) w[e] = f32x2_to_bf16x2(v[2 * e], v[2 * e + 1]);
            else w[e] = __float_as_uint(v[e]);
        }
    }
    __device__ __forceinline__ void store(void* p, int64_t i, int left) const {
        if (left >= 8) {
#pragma unroll
            for (int e = 0; e < WORDS; e += 4) {
                Words* const q = (Words*)((char*)p + i * SIZE) + e / 4;
                const Words v = {w[e], w[e + 1], w[e + 2], w[e + 3]};
                if (POL != kCached && EVEN) __builtin_nontemporal_store(v, q);
                else *q = v;
            }
        } else if (!EVEN) {
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (e < left) {
                    if constexpr (BF16) ((uint16_t*)p)[i + e] = (uint16_t)(w[e / 2] >> (e & 1 ? 16 : 0));
                    else ((uint32_t*)p)[i + e] = w[e];
                }
        }
    }
};

__device__ __forceinline__ void load_floats(float (&v)[8], const float* p, int64_t i, int left, float other) {
    if (p && left >= 8) {
        __builtin_memcpy(v, p + i, sizeof v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = p && e < left ? p[i + e] : other;
    }
}

// Sums over the lanes of a row, K of them at once: `lanes` lanes of a wavefront (a power
// of two), then WAVES wavefronts through LDS, in a fixed order.  The two halves of `lds` take
// turns, so that one barrier a call is enough: a half is written again only behind the
// next call's.
template <int WAVES, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], int lanes, float (*lds)[K][WAVES], int& turn) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        if (WAVES > 1 || m < lanes) {
#pragma unroll
            for (int k = 0; k < K; ++k) v[k] += lanes_xor(v[k], m);
        }
    }
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) lds[turn][k][threadIdx.x >> 6] = v[k];
        }
        barrier_lds();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = lds[turn][k][0];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) v[k] += lds[turn][k][i];
        }
        turn ^= 1;
    }
}

constexpr int threads_of(int waves) { return waves == 1 ? 256 : 64 * waves; }

// Where a thread's octets lie: octet first + 64 WAVES c of the rows row, row + at_once, ...
struct Place {
    int lanes, first;
    int64_t row, at_once, end;          // the workgroup's rows are below `end`
};
template <int WAVES>
__device__ __forceinline__ Place place_of(int64_t n, int64_t d, int64_t rows) {
    Place p;
    const int nv = (int)((d + 7) / 8), lane = threadIdx.x & 63;
    if constexpr (WAVES == 1) {
        p.lanes = nv >= 64 ? 64 : nv <= 1 ? 1 : 1 << (32 - __builtin_clz(nv - 1));
        p.first = lane & (p.lanes - 1);
        p.at_once = 4 * (64 / p.lanes);
        p.row = (threadIdx.x >> 6) * (64 / p.lanes) + lane / p.lanes;
    } else {
        p.lanes = 64;
        p.first = threadIdx.x;
        p.at_once = 1;
        p.row = 0;
    }
    const int64_t from = blockIdx.x * rows * p.at_once;
    p.row += from;
    p.end = from + rows * p.at_once < n ? from + rows * p.at_once : n;
    return p;
}

// A row's values are summed up as 2^-14 of them, which costs no instruction and, above 2^-112,
// changes no digit: the sum of as many as a row may have stays in the range that they are in
constexpr float kSumScale = 0x1p-14f;
static_assert((float)kNormMaxDim * kSumScale <= 1.0f, "the longest rows");

template <bool BF16, bool EVEN, int POL, int WAVES, int CH, int R>
__global__ __launch_bounds__(threads_of(WAVES)) void norm_kernel(NormArgs p) {
    __shared__ float lds[2][R][WAVES];
    int turn = 0;
    const Place at = place_of<WAVES>(p.n, p.d, p.rows);
    DropKey key{};
    if (p.drop.limit) key = drop_key(p.drop);
    float w[CH][8], b[CH][8];
    int left[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t col = 8 * ((int64_t)at.first + 64 * WAVES * c);
        left[c] = p.d - col >= 8 ? 8 : p.d > col ? (int)(p.d - col) : 0;
        load_floats(w[c], p.w, col, left[c], 1.0f);
        load_floats(b[c], p.b, col, left[c], 0.0f);
    }
    // (as many turns for every thread of the workgroup: barriers lie in them)
    for (int64_t base = at.row - at.row % at.at_once; base < at.end; base += R * at.at_once) {
        const int64_t row0 = base + at.row % at.at_once;
        Octet<BF16, EVEN, POL> x[R][CH], res[R][CH];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = row0 + r * at.at_once;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int64_t i = row * p.d + 8 * ((int64_t)at.first + 64 * WAVES * c);
                const int n = row < at.end ? left[c] : 0;
                x[r][c].load(p.x, i, n, p.d >= 8);
                if (p.residual) res[r][c].load(p.residual, i, n, p.d >= 8);
            }
        }
        float s[R][CH][8], sum[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = row0 + r * at.at_once;
            sum[r] = 0.0f;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int64_t col = 8 * ((int64_t)at.first + 64 * WAVES * c);
                const int n = row < at.end ? left[c] : 0;
                x[r][c].settle(n, p.d >= 8);
                x[r][c].values(s[r][c]);
                if (p.drop.limit) drop_octet(s[r][c], key, (uint32_t)(col / 8), (uint32_t)row);
                if (p.residual) {
                    float v[8];
                    res[r][c].settle(n, p.d >= 8);
                    res[r][c].values(v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[r][c][e] += v[e];
                }
                if (p.s) {
                    Octet<BF16, EVEN, POL> o;
                    o.set(s[r][c]);
                    o.store(p.s, row * p.d + col, n);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[r] = __builtin_fmaf(s[r][c][e], kSumScale, sum[r]);
            }
        }
        row_sums<WAVES, R>(sum, at.lanes, lds, turn);
        float mean[R], rstd[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            // (divided, not times 1 / d: a mean that a float holds comes out as it)
            mean[r] = sum[r] / (float)p.d * (1.0f / kSumScale);
            sum[r] = 0.0f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s[r][c][e] = e < left[c] ? s[r][c][e] - mean[r] : 0.0f;
                    sum[r] = __builtin_fmaf(s[r][c][e], s[r][c][e], sum[r]);
                }
        }
        row_sums<WAVES, R>(sum, at.lanes, lds, turn);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = row0 + r * at.at_once;
            rstd[r] = 1.0f / __builtin_sqrtf(sum[r] / (float)p.d + p.eps);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                Octet<BF16, EVEN, POL> o;
#pragma unroll
                for (int e = 0; e < 8; ++e) s[r][c][e] = __builtin_fmaf(s[r][c][e] * rstd[r], w[c][e], b[c][e]);
                o.set(s[r][c]);
                o.store(p.y, row * p.d + 8 * ((int64_t)at.first + 64 * WAVES * c), row < at.end ? left[c] : 0);
            }
            if (p.stats && row < at.end && at.first == 0) {
                p.stats[2 * row] = mean[r];
                p.stats[2 * row + 1] = rstd[r];
            }
        }
    }
}

// What the gradient reads of a lane's place in a row
template <bool BF16, bool EVEN, int POL, int WAVES, int CH>
struct RowIn {
    Octet<BF16, EVEN, POL> x[CH], res[CH], gy[CH], gs[CH];
    float mean, rstd;
    __device__ __forceinline__ void load(const NormBwdArgs& p, const Place& at, int64_t row, const int (&left)[CH]) {
        const bool in = row < at.end;
        mean = in ? p.stats[2 * row] : 0.0f;
        rstd = in ? p.stats[2 * row + 1] : 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t i = row * p.d + 8 * ((int64_t)at.first + 64 * WAVES * c);
            const int n = in ? left[c] : 0;
            x[c].load(p.x, i, n, p.d >= 8);
            if (p.residual) res[c].load(p.residual, i, n, p.d >= 8);
            gy[c].load(p.gy, i, n, p.d >= 8);
            if (p.gs) gs[c].load(p.gs, i, n, p.d >= 8);
        }
    }
};

template <bool BF16, bool EVEN, int POL, int WAVES, int CH>
__global__ __launch_bounds__(threads_of(WAVES)) void norm_bwd_kernel(NormBwdArgs p) {
    __shared__ float lds[2][2][WAVES];
    int turn = 0;
    if (p.hdr && blockIdx.x == 0 && threadIdx.x == 0) {
        p.hdr->timeout = kEmpty32;
        p.hdr->sig = p.sig;
    }
    const Place at = place_of<WAVES>(p.n, p.d, p.rows);
    const float inv = 1.0f / (float)p.d;
    DropKey key{};
    if (p.drop.limit) key = drop_key(p.drop);
    float w[CH][8], dw[CH][8], db[CH][8];
    int left[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t col = 8 * ((int64_t)at.first + 64 * WAVES * c);
        left[c] = p.d - col >= 8 ? 8 : p.d > col ? (int)(p.d - col) : 0;
        load_floats(w[c], p.w, col, left[c], 1.0f);
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[c][e] = db[c][e] = 0.0f;
    }
    // (as many turns for every thread of the workgroup: barriers lie in them)
    const int64_t mine = at.row % at.at_once;
    for (int64_t base = at.row - mine; base < at.end; base += at.at_once) {
        const int64_t row = base + mine;
        RowIn<BF16, EVEN, POL, WAVES, CH> now;
        now.load(p, at, row, left);
        float xh[CH][8], gw[CH][8], sums[2] = {0.0f, 0.0f};
        uint32_t stays[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t col = 8 * ((int64_t)at.first + 64 * WAVES * c);
            const int n = row < at.end ? left[c] : 0;
            now.x[c].settle(n, p.d >= 8);
            now.gy[c].settle(n, p.d >= 8);
            now.x[c].values(xh[c]);
            now.gy[c].values(gw[c]);
            if (p.drop.limit) {
                stays[c] = 0u;
                each_kept(key, (uint32_t)(col / 8), (uint32_t)row, [&](int e, bool on) {
                    xh[c][e] = on ? xh[c][e] * key.scale : 0.0f;
                    stays[c] |= on ? 1u << e : 0u;
                });
            }
            if (p.residual) {
                float v[8];
                now.res[c].settle(n, p.d >= 8);
                now.res[c].values(v);
#pragma unroll
                for (int e = 0; e < 8; ++e) xh[c][e] += v[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float g = gw[c][e], h = e < n ? (xh[c][e] - now.mean) * now.rstd : 0.0f;
                xh[c][e] = h;
                dw[c][e] = __builtin_fmaf(g, h, dw[c][e]);
                db[c][e] += g;
                gw[c][e] = g * w[c][e];
                sums[0] += gw[c][e];
                sums[1] = __builtin_fmaf(gw[c][e], h, sums[1]);
            }
        }
        row_sums<WAVES, 2>(sums, at.lanes, lds, turn);
        const float c1 = sums[0] * inv, c2 = sums[1] * inv;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t i = row * p.d + 8 * ((int64_t)at.first + 64 * WAVES * c);
            const int n = row < at.end ? left[c] : 0;
            float ds[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) ds[e] = now.rstd * (gw[c][e] - c1 - xh[c][e] * c2);
            if (p.gs) {
                float v[8];
                now.gs[c].settle(n, p.d >= 8);
                now.gs[c].values(v);
#pragma unroll
                for (int e = 0; e < 8; ++e) ds[e] += v[e];
            }
            Octet<BF16, EVEN, POL> o;
            if (p.dres) {
                o.set(ds);
                o.store(p.dres, i, n);
            }
            if (p.drop.limit) {
#pragma unroll
                for (int e = 0; e < 8; ++e) ds[e] = stays[c] >> e & 1u ? ds[e] * key.scale : 0.0f;
            }
            o.set(ds);
            o.store(p.dx, i, n);
        }
    }
    if (!p.part) return;
    if constexpr (WAVES == 1) {
        // the rows side by side in a wavefront, then the workgroup's four wavefronts
        __shared__ float sum[3][2][CH * 512];
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            if (m < at.lanes) continue;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    dw[c][e] += lanes_xor(dw[c][e], m);
                    db[c][e] += lanes_xor(db[c][e], m);
                }
        }
        const bool mine = (int)(threadIdx.x & 63) < at.lanes;
        if (wave > 0 && mine) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    sum[wave - 1][0][(c * 8 + e) * 64 + at.first] = dw[c][e];
                    sum[wave - 1][1][(c * 8 + e) * 64 + at.first] = db[c][e];
                }
        }
        barrier_lds();
        if (wave > 0 || !mine) return;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int v = 0; v < 3; ++v) {
                    dw[c][e] += sum[v][0][(c * 8 + e) * 64 + at.first];
                    db[c][e] += sum[v][1][(c * 8 + e) * 64 + at.first];
                }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t col = 8 * ((int64_t)at.first + 64 * WAVES * c);
        float* const o = p.part + 2 * (int64_t)blockIdx.x * p.d + col;
        if (left[c] >= 8) {
            __builtin_memcpy(o, dw[c], sizeof dw[c]);
            __builtin_memcpy(o + p.d, db[c], sizeof db[c]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left[c]) {
                    o[e] = dw[c][e];
                    o[p.d + e] = db[c][e];
                }
        }
    }
}

// dw (blockIdx.y 0) and db (1) from the groups' sums, in doubles: 32 columns, 32 rows at a
// time
__global__ __launch_bounds__(1024) void norm_weights_kernel(const float* part, float* dw, float* db, int64_t groups,
                                                            int64_t d) {
    __shared__ double s[32][32];
    float* const out = blockIdx.y ? db : dw;
    if (!out) return;
    const int col = threadIdx.x & 31, row = threadIdx.x >> 5;
    const int64_t f = (int64_t)blockIdx.x * 32 + col;
    double sum = 0.0;
    if (f < d) {
#pragma unroll 8
        for (int64_t r = row; r < groups; r += 32) sum += (double)part[(2 * r + blockIdx.y) * d + f];
    }
    s[row][col] = sum;
    __syncthreads();
    if (row == 0 && f < d) {
        for (int r = 1; r < 32; ++r) sum += s[r][col];
        out[f] = (float)sum;
    }
}

template <bool BF16, bool EVEN, int POL>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs p) {
    const uint32_t nv = (uint32_t)((p.d + 7) / 8);
    const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (idx >= p.n * nv) return;
    // (idx and nv are below 2^31)
    const uint32_t row = (uint32_t)idx / nv, block = (uint32_t)idx - row * nv;
    const int64_t i = (int64_t)row * p.d + 8 * (int64_t)block;
    const int left = p.d - 8 * (int64_t)block >= 8 ? 8 : (int)(p.d - 8 * (int64_t)block);
    Octet<BF16, EVEN, POL> x, r;
    float v[8];
    x.load(p.x, i, left, p.d >= 8);
    if (p.residual) r.load(p.residual, i, left, p.d >= 8);
    x.settle(left, p.d >= 8);
    x.values(v);
    if (p.drop.limit) drop_octet(v, drop_key(p.drop), block, row);
    if (p.residual) {
        float u[8];
        r.settle(left, p.d >= 8);
        r.values(u);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += u[e];
    }
    x.set(v);
    x.store(p.out, i, left);
}

// Wavefronts of a row, octets of a lane, rows of a workgroup at once.  A lane with one
// octet needs few registers, and workgroups of up to four wavefronts wait for one
// another the least; the longest rows take two octets.  (32768 x 2048 bf16, residual and
// dropout, with four octets a lane and a wavefront a row: 220 and 625 us.)
struct Shape {
    int waves, ch;
    int64_t at_once;
};
Shape shape_of(int64_t d, bool grad) {
    const int64_t nv = (d + 7) / 8;
    int64_t lanes = 1;
    while (lanes < nv && lanes < 64) lanes *= 2;
    if (nv <= 64) return {1, 1, 4 * (64 / lanes)};
    for (int waves = 2; waves <= (grad ? 16 : 8); waves *= 2)
        if (nv <= 64 * waves) return {waves, 1, 1};
    // (16 wavefronts of a row leave no room for another workgroup: 114 us where 8 take 97 at d = 8192)
    if (!grad && nv <= 1024) return {8, 2, 1};
    return {16, 2, 1};
}

template <int W, int C>
struct ShapeOf {
    static constexpr int waves = W, ch = C;
};
template <class F>
void with_shape(const Shape& sh, F&& f) {
    if (sh.ch == 2) {
        if (sh.waves == 8) f(ShapeOf<8, 2>{});
        else f(ShapeOf<16, 2>{});
    } else {
        switch (sh.waves) {
            case 1: f(ShapeOf<1, 1>{}); break;
            case 2: f(ShapeOf<2, 1>{}); break;
            case 4: f(ShapeOf<4, 1>{}); break;
            case 8: f(ShapeOf<8, 1>{}); break;
            default: f(ShapeOf<16, 1>{}); break;
        }
    }
}

// The kinds of rows, and how they go through the caches (CachePolicy, kernels.hpp).  In
// bf16 a lane's octet is one access and a wavefront's whole lines: outputs go past the
// caches, inputs where the tensor is larger than they would be found in later (dropout with a
// residual, 32768 x 2048: 69.2 -> 64.9 us, the norm 107 -> 97, its gradient 166 -> 162).  In fp32 an
// octet is two accesses of every other 16 bytes, which that slows (71 -> 73, 110 -> 117 us); rows
// that are not whole octets share lines, so their outputs stay in the caches.
// With one tensor in and one out neither pays (dropout alone 46.4 -> 49.2 us).
template <class F>
void with_rows(bool bf16, bool few, int64_t n, int64_t d, F&& f) {
    const bool even = d % 8 == 0, large = (double)n * (double)d * 2 > (double)kCachedTensorBytes;
    using std::integral_constant;
    if (!bf16) even ? f(std::false_type{}, std::true_type{}, integral_constant<int, kCached>{})
                    : f(std::false_type{}, std::false_type{}, integral_constant<int, kCached>{});
    else if (!even) f(std::true_type{}, std::false_type{}, integral_constant<int, kStreamAll>{});
    else if (few) f(std::true_type{}, std::true_type{}, integral_constant<int, kCached>{});
    else if (large) f(std::true_type{}, std::true_type{}, integral_constant<int, kStreamAll>{});
    else f(std::true_type{}, std::true_type{}, integral_constant<int, kStreamOut>{});
}

// Rows that a lane sees one after the other, so that about `groups` workgroups of four
// wavefronts, and never a few more, take all: at most 64 (more past 2^26 workgroups of one row a
// lane).  A sum for the weights adds them as floats; where a workgroup has rows side by side,
// the 64 / lanes in a wavefront and then the four wavefronts are floats too.  Over the
// workgroups it goes on in doubles.
int64_t rows_of(int64_t n, const Shape& sh, int64_t groups) {
    const int64_t steps = (n + sh.at_once - 1) / sh.at_once;   // workgroups with a row a lane
    if (sh.waves > 4) groups = groups * 4 / sh.waves;
    int64_t rows = (steps + groups - 1) / groups;
    if (rows > 64) rows = 64 > steps / (1 << 20) ? 64 : steps / (1 << 20);       // (a grid has its limits)
    return rows < 1 ? 1 : rows;
}
int64_t groups_of(int64_t n, const Shape& sh, int64_t rows) { return (n + sh.at_once * rows - 1) / (sh.at_once * rows); }

// The gradient's rows: 1024 workgroups at most run at once, with a row's loads on the way.
// With a residual (and two more tensors to read) half of them do, and leave half as many
// sums.  In us with 512 and 1024, bf16 (fp32): with a residual 262144 x 256 123 and 134 (268 and
// 274), 32768 x 2048 124 and 136 (268 and 277); without 94 and 82 (159 and 165), 101 and 86 (160
// and 168).  Rows that are no whole octets, whose last ones straddle lines, and wide ones,
// whose wavefronts wait for one another, need all of them: with a residual 262144 x 250 187 and
// 150 (302 and 274), 32768 x 2047 198 and 156 (306 and 281), 16384 x 4096 139 and 128 (270 and 271).
int64_t bwd_groups(const Shape& sh, int64_t d, bool residual) {
    return residual && sh.waves <= 4 && d % 8 == 0 ? 512 : 1024;
}

}  // namespace

int64_t norm_groups(int64_t n, int64_t d, bool residual, int64_t* rows) {
    const Shape sh = shape_of(d, true);
    *rows = rows_of(n, sh, bwd_groups(sh, d, residual));
    return groups_of(n, sh, *rows);
}

hipError_t norm_launch(bool bf16, NormArgs a, hipStream_t s) {
    const Shape sh = shape_of(a.d, false);
    // (many more workgroups than run at once: those that end make room; 2048 of them 115 us
    // where 8192 take 97)
    a.rows = rows_of(a.n, sh, 8192);
    with_rows(bf16, !a.residual, a.n, a.d, [&](auto b, auto even, auto pol) {
        with_shape(sh, [&](auto t) {
            using T = decltype(t);
            hipLaunchKernelGGL((norm_kernel<b.value, even.value, pol.value, T::waves, T::ch, T::ch == 1 ? 2 : 1>),
                               dim3((unsigned)groups_of(a.n, sh, a.rows)), dim3(threads_of(T::waves)), 0, s, a);
        });
    });
    return hipGetLastError();
}
hipError_t norm_bwd_launch(bool bf16, const NormBwdArgs& a, hipStream_t s) {
    const Shape sh = shape_of(a.d, true);
    with_rows(bf16, false, a.n, a.d, [&](auto b, auto even, auto pol) {
        with_shape(sh, [&](auto t) {
            using T = decltype(t);
            if constexpr (T::waves != 8 || T::ch == 1)
                hipLaunchKernelGGL((norm_bwd_kernel<b.value, even.value, pol.value, T::waves, T::ch>), dim3((unsigned)a.groups),
                                   dim3(threads_of(T::waves)), 0, s, a);
        });
    });
    if (!a.part) return hipGetLastError();
    hipLaunchKernelGGL(norm_weights_kernel, dim3((unsigned)((a.d + 31) / 32), 2), dim3(1024), 0, s, a.part, a.dw, a.db,
                       a.groups, a.d);
    return hipGetLastError();
}
hipError_t dropout_launch(bool bf16, const DropoutArgs& a, hipStream_t s) {
    with_rows(bf16, !a.residual, a.n, a.d, [&](auto b, auto even, auto pol) {
        hipLaunchKernelGGL((dropout_kernel<b.value, even.value, pol.value>),
                           dim3((unsigned)((a.n * ((a.d + 7) / 8) + 255) / 256)), dim3(256), 0, s, a);
    });
    return hipGetLastError();
}

}  // namespace memoroid
