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
// A lane has octets (eight elements in a row) 64 apart, CH of them; a row takes up to
// a wavefront (the lanes of short rows hold several), four or sixteen.
#include <type_traits>

#include "philox.hpp"

namespace memoroid {

namespace {

// Eight elements in memory order; `left` of them lie in the row.
template <bool BF16>
struct Octet {
    static constexpr int WORDS = BF16 ? 4 : 8;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const void* p, int64_t i, int left) {
        if (left >= 8) {
            // (rows of odd widths start at any element: 16-byte accesses at that
            // alignment, which the hardware takes)
            __builtin_memcpy(w, (const char*)p + i * (BF16 ? 2 : 4), sizeof w);
        } else {
#pragma unroll
            for (int e = 0; e < WORDS; ++e) w[e] = 0u;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (e >= left) break;
                if constexpr (BF16) w[e / 2] |= (uint32_t)((const uint16_t*)p)[i + e] << (e & 1 ? 16 : 0);
                else w[e] = ((const uint32_t*)p)[i + e];
            }
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
            __builtin_memcpy((char*)p + i * (BF16 ? 2 : 4), w, sizeof w);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (e >= left) break;
                if constexpr (BF16) ((uint16_t*)p)[i + e] = (uint16_t)(w[e / 2] >> (e & 1 ? 16 : 0));
                else ((uint32_t*)p)[i + e] = w[e];
            }
        }
    }
};

__device__ __forceinline__ void load_floats(float (&v)[8], const float* p, int64_t i, int left, float other) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = p && e < left ? p[i + e] : other;
}

// Sum over the lanes of a row: lanes of a wavefront (a power of two of them, `lanes`),
// then WAVES wavefronts through LDS, in a fixed order.
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, int lanes, float* lds) {
    for (int m = 1; m < lanes; m <<= 1) v += lanes_xor(v, m);
    if constexpr (WAVES > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) lds[wave] = v;
        barrier_lds();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) v += lds[i];
        barrier_lds();
    }
    return v;
}

template <int WAVES>
constexpr int block_of() { return WAVES == 1 ? 256 : 64 * WAVES; }

// Where a thread's octets lie: octet `first` + 64 WAVES c of row `row` + at_once k
struct Place {
    int lanes, first;
    int64_t row, at_once;
};
template <int WAVES>
__device__ __forceinline__ Place place_of(int64_t d, int64_t rows) {
    Place p;
    const int nv = (int)((d + 7) / 8);
    if constexpr (WAVES == 1) {
        p.lanes = nv >= 64 ? 64 : nv <= 1 ? 1 : 1 << (32 - __builtin_clz(nv - 1));
        const int lane = threadIdx.x & 63;
        p.first = lane & (p.lanes - 1);
        p.at_once = 64 / p.lanes;
        p.row = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * p.at_once * rows + lane / p.lanes;
    } else {
        p.lanes = 64;
        p.first = threadIdx.x;
        p.at_once = 1;
        p.row = (int64_t)blockIdx.x * rows;
    }
    return p;
}

template <bool BF16, int WAVES, int CH>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void norm_kernel(NormArgs p) {
    __shared__ float lds[WAVES];
    const Place at = place_of<WAVES>(p.d, p.rows);
    const float inv = 1.0f / (float)p.d;
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
    for (int64_t k = 0; k < p.rows; ++k) {
        const int64_t row = at.row + at.at_once * k;
        const bool in = row < p.n;             // (uniform where barriers follow: a row is the workgroup's)
        if (WAVES > 1 && !in) return;
        float s[CH][8], sum = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t col = 8 * ((int64_t)at.first + 64 * WAVES * c), i = row * p.d + col;
            const int n = in ? left[c] : 0;
            Octet<BF16> x;
            x.load(p.x, i, n);
            x.values(s[c]);
            if (p.drop.limit) drop_octet(s[c], key, (uint32_t)(col / 8), (uint32_t)row);
            if (p.residual) {
                Octet<BF16> r;
                float v[8];
                r.load(p.residual, i, n);
                r.values(v);
#pragma unroll
                for (int e = 0; e < 8; ++e) s[c][e] += v[e];
            }
            if (p.s) {
                Octet<BF16> o;
                o.set(s[c]);
                o.store(p.s, i, n);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += s[c][e];
        }
        // (divided, not times 1 / d: a mean that a float holds comes out as it)
        const float mean = row_sum<WAVES>(sum, at.lanes, lds) / (float)p.d;
        sum = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s[c][e] = e < left[c] ? s[c][e] - mean : 0.0f;
                sum = __builtin_fmaf(s[c][e], s[c][e], sum);
            }
        const float rstd = 1.0f / __builtin_sqrtf(row_sum<WAVES>(sum, at.lanes, lds) * inv + p.eps);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t i = row * p.d + 8 * ((int64_t)at.first + 64 * WAVES * c);
            Octet<BF16> o;
#pragma unroll
            for (int e = 0; e < 8; ++e) s[c][e] = __builtin_fmaf(s[c][e] * rstd, w[c][e], b[c][e]);
            o.set(s[c]);
            o.store(p.y, i, in ? left[c] : 0);
        }
        if (p.stats && in && at.first == 0) {
            p.stats[2 * row] = mean;
            p.stats[2 * row + 1] = rstd;
        }
    }
}

template <bool BF16, int WAVES, int CH>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void norm_bwd_kernel(NormBwdArgs p) {
    __shared__ float lds[WAVES];
    const Place at = place_of<WAVES>(p.d, p.rows);
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
    for (int64_t k = 0; k < p.rows; ++k) {
        const int64_t row = at.row + at.at_once * k;
        const bool in = row < p.n;
        if (WAVES > 1 && !in) break;
        const float mean = in ? p.stats[2 * row] : 0.0f, rstd = in ? p.stats[2 * row + 1] : 0.0f;
        float xh[CH][8], gy[CH][8], c1 = 0.0f, c2 = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t col = 8 * ((int64_t)at.first + 64 * WAVES * c), i = row * p.d + col;
            const int n = in ? left[c] : 0;
            Octet<BF16> x, g;
            x.load(p.x, i, n);
            g.load(p.gy, i, n);
            x.values(xh[c]);
            g.values(gy[c]);
            if (p.drop.limit) drop_octet(xh[c], key, (uint32_t)(col / 8), (uint32_t)row);
            if (p.residual) {
                Octet<BF16> r;
                float v[8];
                r.load(p.residual, i, n);
                r.values(v);
#pragma unroll
                for (int e = 0; e < 8; ++e) xh[c][e] += v[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                xh[c][e] = e < n ? (xh[c][e] - mean) * rstd : 0.0f;
                dw[c][e] = __builtin_fmaf(gy[c][e], xh[c][e], dw[c][e]);
                db[c][e] += gy[c][e];
                gy[c][e] *= w[c][e];
                c1 += gy[c][e];
                c2 = __builtin_fmaf(gy[c][e], xh[c][e], c2);
            }
        }
        c1 = row_sum<WAVES>(c1, at.lanes, lds) * inv;
        c2 = row_sum<WAVES>(c2, at.lanes, lds) * inv;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t col = 8 * ((int64_t)at.first + 64 * WAVES * c), i = row * p.d + col;
            const int n = in ? left[c] : 0;
            float ds[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) ds[e] = rstd * (gy[c][e] - c1 - xh[c][e] * c2);
            if (p.gs) {
                Octet<BF16> g;
                float v[8];
                g.load(p.gs, i, n);
                g.values(v);
#pragma unroll
                for (int e = 0; e < 8; ++e) ds[e] += v[e];
            }
            Octet<BF16> o;
            if (p.dres) {
                o.set(ds);
                o.store(p.dres, i, n);
            }
            if (p.dx) {
                if (p.drop.limit) drop_octet(ds, key, (uint32_t)(col / 8), (uint32_t)row);
                o.set(ds);
                o.store(p.dx, i, n);
            }
        }
    }
    if (!p.part) return;
    // the sums of a workgroup's wavefronts, then of the rows that one holds side by side
    if constexpr (WAVES == 1) {
        for (int m = at.lanes; m < 64; m <<= 1) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    dw[c][e] += lanes_xor(dw[c][e], m);
                    db[c][e] += lanes_xor(db[c][e], m);
                }
        }
    }
    const int64_t group = WAVES == 1 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
    if (WAVES == 1 && (int)(threadIdx.x & 63) >= at.lanes) return;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t col = 8 * ((int64_t)at.first + 64 * WAVES * c);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left[c]) {
                p.part[(2 * group) * p.d + col + e] = dw[c][e];
                p.part[(2 * group + 1) * p.d + col + e] = db[c][e];
            }
    }
}

// dw (blockIdx.y 0) and db (1) from the groups' sums, in doubles: 64 columns, 16 rows at a time
__global__ __launch_bounds__(1024) void norm_weights_kernel(const float* part, float* dw, float* db, int64_t groups,
                                                            int64_t d) {
    __shared__ double s[16][64];
    float* const out = blockIdx.y ? db : dw;
    if (!out) return;
    const int col = threadIdx.x & 63, row = threadIdx.x >> 6;
    const int64_t f = (int64_t)blockIdx.x * 64 + col;
    double sum = 0.0;
    if (f < d)
        for (int64_t r = row; r < groups; r += 16) sum += (double)part[(2 * r + blockIdx.y) * d + f];
    s[row][col] = sum;
    __syncthreads();
    if (row == 0 && f < d) {
        for (int r = 1; r < 16; ++r) sum += s[r][col];
        out[f] = (float)sum;
    }
}

template <bool BF16>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs p) {
    const int64_t nv = (p.d + 7) / 8, idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (idx >= p.n * nv) return;
    const int64_t row = idx / nv, block = idx - row * nv, i = row * p.d + 8 * block;
    const int left = p.d - 8 * block >= 8 ? 8 : (int)(p.d - 8 * block);
    Octet<BF16> x;
    float v[8];
    x.load(p.x, i, left);
    x.values(v);
    if (p.drop.limit) drop_octet(v, drop_key(p.drop), (uint32_t)block, (uint32_t)row);
    if (p.residual) {
        Octet<BF16> r;
        float u[8];
        r.load(p.residual, i, left);
        r.values(u);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += u[e];
    }
    x.set(v);
    x.store(p.out, i, left);
}

// wavefronts of a row and octets of a lane
struct Shape {
    int waves, ch;
    int64_t at_once;    // rows of a workgroup at once
};
Shape shape_of(int64_t d) {
    const int64_t nv = (d + 7) / 8;
    int64_t lanes = 1;
    while (lanes < nv && lanes < 64) lanes *= 2;
    if (nv <= 64) return {1, 1, 4 * (64 / lanes)};
    if (nv <= 128) return {1, 2, 4};
    if (nv <= 256) return {1, 4, 4};
    if (nv <= 512) return {4, 2, 1};
    if (nv <= 1024) return {4, 4, 1};
    return {16, 2, 1};
}

template <bool BF16, class F>
hipError_t with_shape(const Shape& sh, F&& f) {
    if (sh.waves == 1 && sh.ch == 1) f(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{});
    else if (sh.waves == 1 && sh.ch == 2) f(std::integral_constant<int, 1>{}, std::integral_constant<int, 2>{});
    else if (sh.waves == 1) f(std::integral_constant<int, 1>{}, std::integral_constant<int, 4>{});
    else if (sh.waves == 4 && sh.ch == 2) f(std::integral_constant<int, 4>{}, std::integral_constant<int, 2>{});
    else if (sh.waves == 4) f(std::integral_constant<int, 4>{}, std::integral_constant<int, 4>{});
    else f(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
    return hipGetLastError();
}

int64_t rows_of(int64_t n, const Shape& sh, int64_t most) {
    const int64_t steps = (n + sh.at_once - 1) / sh.at_once;   // workgroups with a row each
    int64_t rows = steps / 1024;
    if (rows > most) rows = most > steps / (1 << 20) ? most : steps / (1 << 20);   // (a grid has its limits)
    return rows < 1 ? 1 : rows;
}

template <bool BF16>
hipError_t norm_launch_t(NormArgs a, hipStream_t s) {
    const Shape sh = shape_of(a.d);
    a.rows = rows_of(a.n, sh, 16);
    const dim3 grid((unsigned)((a.n + sh.at_once * a.rows - 1) / (sh.at_once * a.rows)));
    return with_shape<BF16>(sh, [&](auto waves, auto ch) {
        hipLaunchKernelGGL((norm_kernel<BF16, waves.value, ch.value>), grid, dim3(block_of<waves.value>()), 0, s, a);
    });
}
template <bool BF16>
hipError_t norm_bwd_launch_t(NormBwdArgs a, hipStream_t s) {
    const Shape sh = shape_of(a.d);
    const dim3 grid((unsigned)((a.n + sh.at_once * a.rows - 1) / (sh.at_once * a.rows)));
    const hipError_t e = with_shape<BF16>(sh, [&](auto waves, auto ch) {
        hipLaunchKernelGGL((norm_bwd_kernel<BF16, waves.value, ch.value>), grid, dim3(block_of<waves.value>()), 0, s, a);
    });
    if (e != hipSuccess || !a.part) return e;
    hipLaunchKernelGGL(norm_weights_kernel, dim3((unsigned)((a.d + 63) / 64), 2), dim3(1024), 0, s, a.part, a.dw, a.db,
                       a.groups, a.d);
    return hipGetLastError();
}

}  // namespace

int64_t norm_groups(int64_t n, int64_t d, int64_t* rows) {
    const Shape sh = shape_of(d);
    *rows = rows_of(n, sh, 64);
    const int64_t blocks = (n + sh.at_once * *rows - 1) / (sh.at_once * *rows);
    return sh.waves == 1 ? 4 * blocks : blocks;
}

hipError_t norm_launch(bool bf16, NormArgs a, hipStream_t s) {
    return bf16 ? norm_launch_t<true>(a, s) : norm_launch_t<false>(a, s);
}
hipError_t norm_bwd_launch(bool bf16, NormBwdArgs a, hipStream_t s) {
    return bf16 ? norm_bwd_launch_t<true>(a, s) : norm_bwd_launch_t<false>(a, s);
}
hipError_t dropout_launch(bool bf16, const DropoutArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)((a.n * ((a.d + 7) / 8) + 255) / 256));
    if (bf16) hipLaunchKernelGGL(dropout_kernel<true>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(dropout_kernel<false>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace memoroid
