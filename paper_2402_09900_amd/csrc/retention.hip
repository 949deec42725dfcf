// retention.hip -- kernels of the retention operator and its gradient for
// gfx950: linear attention over tapes of episodes whose state decays at a rate
// of its own in each head.  retention_common.hpp has the walk W(x, y, z) that
// all of them are, and the layouts.
//
// Per chunk of C rows with the state S before it, e = 1, first(i) the first row
// of row i's episode in the chunk:
//     P_ij = gamma^(i-j) x_i . y_j            first(i) <= j <= i, 0 elsewhere
//     W_i  = sum_j P_ij z_j + gamma^(i+e) x_i S   (S only where i's episode began earlier)
//     S'   = gamma^(n-1+e) S + sum_j gamma^(n-1-j) y_j^T z_j   (rows from the last begin on)
// The walks backwards start from the gradient of the state after the tape, which
// belongs to the last step itself: e = 0 in their first chunk.
//
// Precision.  States, decays and all sums are floats; z is multiplied by its
// decay in float and goes into the state as three planes, exactly.  With bf16
// inputs P and the S that a row is multiplied with are rounded to bf16 once
// each, as operands: together they add to the output's own rounding what one
// more rounding would (1.4 times its error), and the state itself takes neither.
//
// A value that is not finite must not reach other episodes, nor earlier rows of
// its own, through a zero of P or of the decays (0 * NaN): a chunk that holds one
// is walked row by row, each a chunk of its own with the other rows as zeros.
#include "retention_common.hpp"

namespace memoroid {

__device__ __forceinline__ void ret_header(WsHeader* hdr, uint64_t sig) {
    if (hdr && blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x < 16) {
        const u32x4 ones = {kEmpty32, kEmpty32, kEmpty32, kEmpty32};
        const u32x4 head = {kEmpty32, kEmpty32, (uint32_t)sig, (uint32_t)(sig >> 32)};
        ((u32x4*)hdr)[threadIdx.x] = threadIdx.x == 0 ? head : ones;
    }
}

template <int ES>
__device__ __forceinline__ const void* role_head(const RetRole& x, int64_t b, int64_t h, int64_t T) {
    return (const char*)x.p + (b * T * x.heads + h / x.share) * x.d * ES;
}

template <class Cfg>
using State = f32x4[Cfg::KD / 32][2][Cfg::NT];

template <class Cfg>
__device__ __forceinline__ void zero_state(State<Cfg>& S) {
#pragma unroll
    for (int s = 0; s < Cfg::KD / 32; ++s)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int nt = 0; nt < Cfg::NT; ++nt) S[s][u][nt] = zero4();
}
template <class Cfg>
__device__ __forceinline__ void carry_state(State<Cfg>& S, const Carry& cy, bool drop) {
#pragma unroll
    for (int s = 0; s < Cfg::KD / 32; ++s)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int nt = 0; nt < Cfg::NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) S[s][u][nt][e] = drop ? 0.0f : cy(S[s][u][nt][e]);
}
// the value operand times a weight per row, in planes
template <class Cfg>
__device__ __forceinline__ void weigh(bf16x8 (&out)[3], const bf16x8 (&z)[Cfg::NP], const float* w, int tb,
                                      const RetLane& L) {
    f32x4 lo = *(const f32x4*)(w + 32 * tb + 4 * L.g), hi = *(const f32x4*)(w + 32 * tb + 16 + 4 * L.g);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        lo[e] *= plane_value<Cfg::NP>(z, e);
        hi[e] *= plane_value<Cfg::NP>(z, e + 4);
    }
    planes8<3>(lo, hi, out);
}
// S += y^T (weighted z) over rows 32 tb .. + 31
template <class Cfg>
__device__ __forceinline__ void state_add(State<Cfg>& S, const uint16_t* sY, const bf16x8 (&zw)[Cfg::NT][3], int tb,
                                          const RetLane& L) {
#pragma unroll
    for (int s = 0; s < Cfg::KD / 32; ++s)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            bf16x8 y[Cfg::NP];
            col_frag<Cfg, Cfg::LDK>(y, sY, tb, state_row_addr<Cfg>(s, u, L), L);
#pragma unroll
            for (int nt = 0; nt < Cfg::NT; ++nt) mma<Cfg::NP, 3>(S[s][u][nt], y, zw[nt]);
        }
}
// tile `idx` of the triangle: rows 16 jb.. of y against rows 16 ib.. of x
__device__ __forceinline__ void tile_of(int idx, int& jb, int& ib) {
    ib = idx >= 6 ? 3 : idx >= 3 ? 2 : idx >= 1 ? 1 : 0;
    jb = idx - ib * (ib + 1) / 2;
}
template <class Cfg, int LD, int D>
__device__ __forceinline__ f32x4 pair_products(const uint16_t* sY, const uint16_t* sX, int jb, int ib, const RetLane& L) {
    f32x4 d = zero4();
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
        bf16x8 y[Cfg::NP], x[Cfg::NP];
        row_frag<Cfg, LD>(y, sY, 16 * jb, 32 * s, L);
        row_frag<Cfg, LD>(x, sX, 16 * ib, 32 * s, L);
        mma<Cfg::NP, Cfg::NP>(d, y, x);
    }
    return d;
}

// ---------------------------------------------------------------- summaries
// What a segment adds to the state after it: the sum over its rows from the last
// begin on.  DOT: also its derivative by log gamma, sum (n-1-j) gamma^(n-1-j) y^T z.
template <class Cfg, bool DOT>
__global__ __launch_bounds__(256, 2) void ret_summary_kernel(RetSummaryArgs p) {
    __shared__ __attribute__((aligned(16))) uint16_t sY[Cfg::NP * Cfg::C * Cfg::LDK];
    __shared__ __attribute__((aligned(16))) uint16_t sZ[Cfg::NP * Cfg::C * Cfg::LDV];
    __shared__ float sPw[Cfg::C + 1];
    __shared__ __attribute__((aligned(16))) float sW[DOT ? 2 : 1][Cfg::C];
    const RetLane L;
    const int64_t seg = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    ret_header(p.hdr, p.sig);
    const double rate = fabs((double)p.alpha[h]);
    if (L.tid <= Cfg::C) sPw[L.tid] = decay_pow(rate, L.tid);
    const Carry full = carry_of(rate, Cfg::C);
    const void* const y0 = role_head<Cfg::ES>(p.y, b, h, p.T);
    const void* const z0 = role_head<Cfg::ES>(p.z, b, h, p.T);
    const int64_t yrow = (int64_t)p.y.heads * p.y.d, zrow = (int64_t)p.z.heads * p.z.d;
    const uint8_t* const start = p.start + b * p.T;
    State<Cfg> S, D;
    zero_state<Cfg>(S);
    if (DOT) zero_state<Cfg>(D);
    bool any = false;
    RetTile<Cfg, Cfg::KD> ty;
    RetTile<Cfg, Cfg::VD> tz;
#pragma unroll 1
    for (int ch = 0; ch < p.chunks; ++ch) {
        // every segment here is a whole one: C rows per chunk
        const int64_t w0 = (seg * p.chunks + ch) * Cfg::C;
        ty.fetch(ret_rows<Cfg::ES>(y0, yrow, p.y.d, w0, Cfg::C, p.T, p.rev), L);
        tz.fetch(ret_rows<Cfg::ES>(z0, zrow, p.z.d, w0, Cfg::C, p.T, p.rev), L);
        const uint64_t m = ret_begins(start, w0, Cfg::C, p.T, p.rev, L.lane);
        const int from = m ? last_begin(m) : 0;
        any = any || m != 0;
        __syncthreads();                                   // the last chunk's operands have been read
        ty.template stage<Cfg::LDK>(sY, from, Cfg::C, L);
        tz.template stage<Cfg::LDV>(sZ, from, Cfg::C, L);
        if (L.tid < Cfg::C) {
            const int age = Cfg::C - 1 - L.tid;
            const float w = L.tid >= from ? sPw[age] * p.z_scale : 0.0f;
            sW[0][L.tid] = w;
            if (DOT) sW[DOT ? 1 : 0][L.tid] = w * (float)age;
        }
        __syncthreads();
        if (DOT) {
            // d(gamma^C S)/dlog gamma = gamma^C (D + C S)
#pragma unroll
            for (int s = 0; s < Cfg::KD / 32; ++s)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int nt = 0; nt < Cfg::NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            D[s][u][nt][e] = __builtin_fmaf((float)Cfg::C, S[s][u][nt][e], D[s][u][nt][e]);
            carry_state<Cfg>(D, full, m != 0);
        }
        carry_state<Cfg>(S, full, m != 0);
#pragma unroll
        for (int tb = 0; tb < Cfg::C / 32; ++tb) {
            bf16x8 z[Cfg::NT][Cfg::NP], zw[Cfg::NT][3];
#pragma unroll
            for (int nt = 0; nt < Cfg::NT; ++nt) {
                col_frag<Cfg, Cfg::LDV>(z[nt], sZ, tb, state_col_addr<Cfg>(nt, L), L);
                weigh<Cfg>(zw[nt], z[nt], sW[0], tb, L);
            }
            state_add<Cfg>(S, sY, zw, tb, L);
            if (DOT) {
#pragma unroll
                for (int nt = 0; nt < Cfg::NT; ++nt) weigh<Cfg>(zw[nt], z[nt], sW[DOT ? 1 : 0], tb, L);
                state_add<Cfg>(D, sY, zw, tb, L);
            }
        }
    }
    const int64_t words = (int64_t)p.y.d * p.z.d, n = p.nseg - 1;
    const int64_t at = ((b * p.H + h) * n + seg) * words;
    store_state<Cfg>(S, p.states + at, p.z.d, 1, p.y.d, p.z.d, 1.0f, false, L);
    if (DOT) store_state<Cfg>(D, p.dstates + at, p.z.d, 1, p.y.d, p.z.d, 1.0f, false, L);
    if (h == 0 && L.tid == 0) p.R[b * n + seg] = any ? 1 : 0;
}

// ---------------------------------------------------------------- state scan
// states[i] becomes the state after segment i: its summary, plus gamma^rows times
// the state before it where it holds no begin step.
template <bool DOT>
__global__ __launch_bounds__(256) void ret_state_scan_kernel(RetStateScanArgs p) {
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x, h = blockIdx.y, b = blockIdx.z;
    if (e >= p.words) return;
    const double rate = fabs((double)p.alpha[h]);
    const int64_t bh = b * p.H + h;
    const Carry full = carry_of(rate, (double)p.rows);
    float s = p.seed ? p.seed[bh * p.words + e] : 0.0f, d = 0.0f;
    float* const at = p.states + bh * p.n * p.words + e;
    float* const dat = DOT ? p.dstates + bh * p.n * p.words + e : nullptr;
    const uint8_t* const R = p.R + b * p.n;
#pragma unroll 4
    for (int i = 0; i < p.n; ++i) {
        const float own = at[(int64_t)i * p.words], down = DOT ? dat[(int64_t)i * p.words] : 0.0f;
        const Carry cy = i == 0 && p.rev ? carry_of(rate, (double)(p.rows - 1)) : full;
        if (DOT) d = down + (R[i] ? 0.0f : cy(__builtin_fmaf((float)p.rows, s, d)));
        s = own + (R[i] ? 0.0f : cy(s));
        at[(int64_t)i * p.words] = s;
        if (DOT) dat[(int64_t)i * p.words] = d;
    }
}

// ---------------------------------------------------------------------- walk
template <class Cfg>
__global__ __launch_bounds__(256, Cfg::NP == 1 ? 2 : 1) void ret_walk_kernel(RetWalkArgs p) {
    __shared__ __attribute__((aligned(16))) uint16_t sX[Cfg::NP * Cfg::C * Cfg::LDK];
    __shared__ __attribute__((aligned(16))) uint16_t sY[Cfg::NP * Cfg::C * Cfg::LDK];
    __shared__ __attribute__((aligned(16))) uint16_t sZ[Cfg::NP * Cfg::C * Cfg::LDV];
    __shared__ u32x2 sP[Cfg::NTILE][Cfg::NP][64];
    __shared__ float sPw[Cfg::C + 1];
    __shared__ __attribute__((aligned(16))) float sW[Cfg::C];
    __shared__ uint32_t sBad[4];
    const RetLane L;
    const int64_t seg = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    ret_header(p.hdr, p.sig);
    const double rate = fabs((double)p.alpha[h]);
    if (L.tid <= Cfg::C) sPw[L.tid] = decay_pow(rate, L.tid);
    const Carry full = carry_of(rate, Cfg::C);
    const void* const x0 = role_head<Cfg::ES>(p.x, b, h, p.T);
    const void* const y0 = role_head<Cfg::ES>(p.y, b, h, p.T);
    const void* const z0 = role_head<Cfg::ES>(p.z, b, h, p.T);
    const int64_t xrow = (int64_t)p.x.heads * p.x.d, yrow = (int64_t)p.y.heads * p.y.d;
    const int64_t zrow = (int64_t)p.z.heads * p.z.d, orow = (int64_t)p.H * p.z.d;
    const uint8_t* const start = p.start + b * p.T;
    const int64_t words = (int64_t)p.x.d * p.z.d, bh = b * p.H + h;
    const int64_t seg0 = seg * p.chunks * Cfg::C;
    const int64_t left = (p.T - seg0 + Cfg::C - 1) / Cfg::C;
    const int nch = (int)(left < p.chunks ? left : p.chunks);

    State<Cfg> S;
    const float* const before = seg == 0 ? (p.seed ? p.seed + bh * words : nullptr)
                                         : p.states + (bh * (p.nseg - 1) + seg - 1) * words;
    load_state<Cfg>(S, before, p.sk, p.sv, p.x.d, p.z.d, L);

    RetTile<Cfg, Cfg::KD> tx, ty;
    RetTile<Cfg, Cfg::VD> tz;
    auto fetch = [&](int ch) {
        const int64_t w0 = seg0 + (int64_t)ch * Cfg::C;
        const int64_t rest = ch < nch ? p.T - w0 : 0;
        const int n = (int)(rest < Cfg::C ? rest : Cfg::C);
        const int64_t w = ch < nch ? w0 : 0;
        tx.fetch(ret_rows<Cfg::ES>(x0, xrow, p.x.d, w, n, p.T, p.rev), L);
        ty.fetch(ret_rows<Cfg::ES>(y0, yrow, p.y.d, w, n, p.T, p.rev), L);
        tz.fetch(ret_rows<Cfg::ES>(z0, zrow, p.z.d, w, n, p.T, p.rev), L);
    };
    fetch(0);
#pragma unroll 1
    for (int ch = 0; ch < nch; ++ch) {
        const int64_t w0 = seg0 + (int64_t)ch * Cfg::C;
        const int n = (int)(p.T - w0 < Cfg::C ? p.T - w0 : Cfg::C);
        const uint64_t m = ret_begins(start, w0, n, p.T, p.rev, L.lane);
        const uint64_t not_finite = __ballot(tx.bad() || ty.bad() || tz.bad());
        __syncthreads();                                   // the last chunk's operands have been read
        if (L.lane == 0) sBad[L.w] = not_finite != 0;
        tx.template stage<Cfg::LDK>(sX, 0, n, L);
        ty.template stage<Cfg::LDK>(sY, 0, n, L);
        tz.template stage<Cfg::LDV>(sZ, 0, n, L);
        // weights of the rows into the state: no begin step after them
        if (L.tid < Cfg::C) {
            const int from = m ? last_begin(m) : 0;
            sW[L.tid] = L.tid >= from && L.tid < n ? sPw[n - 1 - L.tid] * p.z_scale : 0.0f;
        }
        __syncthreads();
        const bool by_row = (sBad[0] | sBad[1] | sBad[2] | sBad[3]) != 0;
        int a = 0;
#pragma unroll 1
        do {
            const int to = by_row ? a + 1 : n;             // rows a .. to - 1
            if (by_row) {
                __syncthreads();
                tx.template stage<Cfg::LDK>(sX, a, to, L);
                ty.template stage<Cfg::LDK>(sY, a, to, L);
                tz.template stage<Cfg::LDV>(sZ, a, to, L);
                if (L.tid < Cfg::C) sW[L.tid] = L.tid == a ? p.z_scale : 0.0f;
                __syncthreads();
            }
            if (to == n) fetch(ch + 1);
            const uint64_t mw = m & (upto(to - 1) & ~((1ull << a) - 1ull));
            const int e = p.rev && w0 + a == 0 ? 0 : 1;

            // ---- the pairs' products, a few tiles per wavefront
#pragma unroll
            for (int i = 0; i < (Cfg::NTILE + 3) / 4; ++i) {
                const int idx = 4 * i + L.w;
                if (idx >= Cfg::NTILE) break;
                int jb, ib;
                tile_of(idx, jb, ib);
                f32x4 d = pair_products<Cfg, Cfg::LDK, Cfg::KD>(sY, sX, jb, ib, L);
                const int row = 16 * ib + L.c;
                const uint64_t mr = mw & upto(row);
                const int first = mr ? last_begin(mr) : a;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = 16 * jb + 4 * L.g + r;
                    d[r] = j <= row && j >= first ? d[r] * (sPw[j <= row ? row - j : 0] * p.p_scale) : 0.0f;
                }
                uint32_t lo[Cfg::NP], hi[Cfg::NP];
                planes2<Cfg::NP>(d[0], d[1], lo);
                planes2<Cfg::NP>(d[2], d[3], hi);
#pragma unroll
                for (int q = 0; q < Cfg::NP; ++q) sP[idx][q][L.lane] = u32x2{lo[q], hi[q]};
            }
            __syncthreads();

            // ---- the rows against the state before the chunk
            f32x4 acc[Cfg::NB][Cfg::NT];
#pragma unroll
            for (int ib = 0; ib < Cfg::NB; ++ib)
#pragma unroll
                for (int nt = 0; nt < Cfg::NT; ++nt) acc[ib][nt] = zero4();
#pragma unroll
            for (int s = 0; s < Cfg::KD / 32; ++s) {
                bf16x8 st[Cfg::NT][Cfg::NP];
#pragma unroll
                for (int nt = 0; nt < Cfg::NT; ++nt) planes8<Cfg::NP>(S[s][0][nt], S[s][1][nt], st[nt]);
#pragma unroll
                for (int ib = 0; ib < Cfg::NB; ++ib) {
                    bf16x8 x[Cfg::NP];
                    row_frag<Cfg, Cfg::LDK>(x, sX, 16 * ib, 32 * s, L);
#pragma unroll
                    for (int nt = 0; nt < Cfg::NT; ++nt) mma<Cfg::NP, Cfg::NP>(acc[ib][nt], st[nt], x);
                }
            }
#pragma unroll
            for (int ib = 0; ib < Cfg::NB; ++ib) {
                const int row = 16 * ib + L.c;
                const bool goes_on = (mw & upto(row)) == 0 && row >= a && row < to;
                const float f = goes_on ? sPw[row - a + e] * p.inter_scale : 0.0f;
#pragma unroll
                for (int nt = 0; nt < Cfg::NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[ib][nt][r] = goes_on ? acc[ib][nt][r] * f : 0.0f;
            }

            // ---- the rows against each other, and the state after the chunk
            carry_state<Cfg>(S, to - a - 1 + e == Cfg::C ? full : carry_of(rate, (double)(to - a - 1 + e)), mw != 0);
#pragma unroll
            for (int tb = 0; tb < Cfg::C / 32; ++tb) {
                bf16x8 z[Cfg::NT][Cfg::NP], zw[Cfg::NT][3];
#pragma unroll
                for (int nt = 0; nt < Cfg::NT; ++nt)
                    col_frag<Cfg, Cfg::LDV>(z[nt], sZ, tb, state_col_addr<Cfg>(nt, L), L);
#pragma unroll
                for (int ib = 2 * tb; ib < Cfg::NB; ++ib) {
                    const int t0 = ib * (ib + 1) / 2 + 2 * tb;
                    bf16x8 pr[Cfg::NP];
#pragma unroll
                    for (int q = 0; q < Cfg::NP; ++q) {
                        const u32x2 lo = sP[t0][q][L.lane];
                        const u32x2 hi = ib > 2 * tb ? sP[t0 + (ib > 2 * tb ? 1 : 0)][q][L.lane] : u32x2{0u, 0u};
                        pr[q] = __builtin_bit_cast(bf16x8, u32x4{lo.x, lo.y, hi.x, hi.y});
                    }
#pragma unroll
                    for (int nt = 0; nt < Cfg::NT; ++nt) mma<Cfg::NP, Cfg::NP>(acc[ib][nt], z[nt], pr);
                }
#pragma unroll
                for (int nt = 0; nt < Cfg::NT; ++nt) weigh<Cfg>(zw[nt], z[nt], sW, tb, L);
                state_add<Cfg>(S, sY, zw, tb, L);
            }

            // ---- out: 4 NT consecutive columns of a row per lane
            {
                const int os = Cfg::NP == 1 && !p.out_f32 ? 2 : 4;
                const int64_t t = p.rev ? p.T - w0 - n : w0;
                const RetRows o{make_rsrc((char*)p.out + (((b * p.T + t) * p.H + h) * p.z.d) * os,
                                          ((int64_t)(n - 1) * orow + p.z.d) * os),
                                (uint32_t)(orow * os), n, p.z.d, (bool)p.rev};
#pragma unroll
                for (int ib = 0; ib < Cfg::NB; ++ib) {
                    const int row = 16 * ib + L.c;
                    const int col = 16 * Cfg::NT * L.w + 4 * Cfg::NT * L.g;
                    const bool in = row >= a && row < to;
                    const uint32_t off = in ? o.offset(row, col, os) : kOob;
                    if (os == 2) {
                        uint32_t wd[2 * Cfg::NT];
#pragma unroll
                        for (int nt = 0; nt < Cfg::NT; ++nt) {
                            wd[2 * nt] = f32x2_to_bf16x2(acc[ib][nt][0], acc[ib][nt][1]);
                            wd[2 * nt + 1] = f32x2_to_bf16x2(acc[ib][nt][2], acc[ib][nt][3]);
                        }
                        if constexpr (Cfg::NT == 2)
                            __builtin_amdgcn_raw_buffer_store_b128(u32x4{wd[0], wd[1], wd[2], wd[3]}, o.r, (int)off, 0, 0);
                        else
                            __builtin_amdgcn_raw_buffer_store_b64(u32x2{wd[0], wd[1]}, o.r, (int)off, 0, 0);
                    } else {
#pragma unroll
                        for (int nt = 0; nt < Cfg::NT; ++nt)
                            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[ib][nt]), o.r,
                                                                   (int)(off + 16u * nt), 0, 0);
                    }
                }
            }
            a = to;
        } while (a < n);
    }
    if (p.fin && seg == p.nseg - 1) {
        // backwards: the gradient of the state before the tape, one step further
        // back, and none if step 0 begins an episode
        const bool drop = p.rev && start[0] != 0;
        store_state<Cfg>(S, p.fin + bh * words, p.sk, p.sv, p.x.d, p.z.d, p.rev ? decay_pow(rate, 1.0) : 1.0f, drop, L);
    }
}

// ------------------------------------------------------- gradient of the rate
// With D_t = dS_t / dlog gamma, D_t = gamma (D_{t-1} + S_{t-1}) inside an episode,
//     dL/dlog gamma = scale sum_t q_t D_t dout_t^T  (+ D_T-1 . grad_state),
// per chunk, (S, D) before it:
//     sum_ij (i-j) gamma^(i-j) (q_i . k_j)(dout_i . v_j)     both products in float
//   + S . sum_i (i+1) gamma^(i+1) q_i^T dout_i + D . sum_i gamma^(i+1) q_i^T dout_i
// The two outer products arrive in the state's own layout, so they meet S and D
// as floats in registers: nothing here is rounded to bf16.
template <class Cfg>
__global__ __launch_bounds__(256, 1) void ret_sens_kernel(RetSensArgs p) {
    __shared__ __attribute__((aligned(16))) uint16_t sQ[Cfg::NP * Cfg::C * Cfg::LDK];
    __shared__ __attribute__((aligned(16))) uint16_t sK[Cfg::NP * Cfg::C * Cfg::LDK];
    __shared__ __attribute__((aligned(16))) uint16_t sV[Cfg::NP * Cfg::C * Cfg::LDV];
    __shared__ __attribute__((aligned(16))) uint16_t sG[Cfg::NP * Cfg::C * Cfg::LDV];
    __shared__ float sPw[Cfg::C + 1];
    __shared__ __attribute__((aligned(16))) float sW[4][Cfg::C];
    __shared__ uint32_t sBad[4];
    __shared__ double sSum[4];
    const RetLane L;
    const int64_t seg = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    const double rate = fabs((double)p.alpha[h]);
    if (L.tid <= Cfg::C) sPw[L.tid] = decay_pow(rate, L.tid);
    const Carry full = carry_of(rate, Cfg::C);
    const int kd = p.q.d, vd = p.v.d;
    const void* const q0 = role_head<Cfg::ES>(p.q, b, h, p.T);
    const void* const k0 = role_head<Cfg::ES>(p.k, b, h, p.T);
    const void* const v0 = role_head<Cfg::ES>(p.v, b, h, p.T);
    const void* const g0 = role_head<Cfg::ES>(p.g, b, h, p.T);
    const int64_t qrow = (int64_t)p.q.heads * kd, krow = (int64_t)p.k.heads * kd;
    const int64_t vrow = (int64_t)p.v.heads * vd, grow = (int64_t)p.g.heads * vd;
    const uint8_t* const start = p.start + b * p.T;
    const int64_t words = (int64_t)kd * vd, bh = b * p.H + h;
    const int64_t seg0 = seg * p.chunks * Cfg::C;
    const int64_t left = (p.T - seg0 + Cfg::C - 1) / Cfg::C;
    const int nch = (int)(left < p.chunks ? left : p.chunks);

    State<Cfg> S, D;
    const int64_t at = (bh * (p.nseg - 1) + seg - 1) * words;
    load_state<Cfg>(S, seg == 0 ? (p.seed ? p.seed + bh * words : nullptr) : p.states + at, vd, 1, kd, vd, L);
    load_state<Cfg>(D, seg == 0 ? nullptr : p.dstates + at, vd, 1, kd, vd, L);
    double sum = 0.0;
    RetTile<Cfg, Cfg::KD> tq, tk;
    RetTile<Cfg, Cfg::VD> tv, tg;
#pragma unroll 1
    for (int ch = 0; ch < nch; ++ch) {
        const int64_t w0 = seg0 + (int64_t)ch * Cfg::C;
        const int n = (int)(p.T - w0 < Cfg::C ? p.T - w0 : Cfg::C);
        tq.fetch(ret_rows<Cfg::ES>(q0, qrow, kd, w0, n, p.T, false), L);
        tk.fetch(ret_rows<Cfg::ES>(k0, krow, kd, w0, n, p.T, false), L);
        tv.fetch(ret_rows<Cfg::ES>(v0, vrow, vd, w0, n, p.T, false), L);
        tg.fetch(ret_rows<Cfg::ES>(g0, grow, vd, w0, n, p.T, false), L);
        const uint64_t m = ret_begins(start, w0, n, p.T, false, L.lane);
        const uint64_t not_finite = __ballot(tq.bad() || tk.bad() || tv.bad() || tg.bad());
        if (L.lane == 0) sBad[L.w] = not_finite != 0;
        __syncthreads();
        const bool by_row = (sBad[0] | sBad[1] | sBad[2] | sBad[3]) != 0;
        int a = 0;
#pragma unroll 1
        do {
            const int to = by_row ? a + 1 : n;
            const uint64_t mw = m & (upto(to - 1) & ~((1ull << a) - 1ull));
            __syncthreads();                               // the last operands have been read
            tq.template stage<Cfg::LDK>(sQ, a, to, L);
            tk.template stage<Cfg::LDK>(sK, a, to, L);
            tv.template stage<Cfg::LDV>(sV, a, to, L);
            tg.template stage<Cfg::LDV>(sG, a, to, L);
            if (L.tid < Cfg::C) {
                const int i = L.tid;
                const bool in = i >= a && i < to;
                const int from = mw ? last_begin(mw) : a;
                const float w = in && i >= from ? sPw[to - 1 - i] : 0.0f;
                sW[0][i] = w;
                sW[1][i] = w * (float)(to - 1 - i);
                const float f = in && (mw & upto(i)) == 0 ? sPw[i - a + 1] * p.scale : 0.0f;
                sW[2][i] = f;
                sW[3][i] = f * (float)(i - a + 1);
            }
            __syncthreads();
            float part = 0.0f;
#pragma unroll
            for (int i = 0; i < (Cfg::NTILE + 3) / 4; ++i) {
                const int idx = 4 * i + L.w;
                if (idx >= Cfg::NTILE) break;
                int jb, ib;
                tile_of(idx, jb, ib);
                const f32x4 x = pair_products<Cfg, Cfg::LDK, Cfg::KD>(sK, sQ, jb, ib, L);
                const f32x4 y = pair_products<Cfg, Cfg::LDV, Cfg::VD>(sV, sG, jb, ib, L);
                const int row = 16 * ib + L.c;
                const uint64_t mr = mw & upto(row);
                const int first = mr ? last_begin(mr) : a;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = 16 * jb + 4 * L.g + r;
                    const bool in = j < row && j >= first;
                    const float w = sPw[in ? row - j : 0] * (float)(row - j) * p.scale;
                    part += in ? x[r] * y[r] * w : 0.0f;
                }
            }
            // rows against (S, D): skipped where the first row begins an episode,
            // so that values of S that are not finite stay out
            if (!(mw >> a & 1ull)) {
                // two running sums per wavefront column and state row block, in
                // float within the chunk
#pragma unroll 1
                for (int s = 0; s < Cfg::KD / 32; ++s) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        f32x4 o1[Cfg::NT], o2[Cfg::NT];
#pragma unroll
                        for (int nt = 0; nt < Cfg::NT; ++nt) o1[nt] = o2[nt] = zero4();
#pragma unroll
                        for (int tb = 0; tb < Cfg::C / 32; ++tb) {
                            bf16x8 q[Cfg::NP];
                            col_frag<Cfg, Cfg::LDK>(q, sQ, tb, state_row_addr<Cfg>(s, u, L), L);
#pragma unroll
                            for (int nt = 0; nt < Cfg::NT; ++nt) {
                                bf16x8 g[Cfg::NP], gw[3];
                                col_frag<Cfg, Cfg::LDV>(g, sG, tb, state_col_addr<Cfg>(nt, L), L);
                                weigh<Cfg>(gw, g, sW[2], tb, L);
                                mma<Cfg::NP, 3>(o1[nt], q, gw);
                                weigh<Cfg>(gw, g, sW[3], tb, L);
                                mma<Cfg::NP, 3>(o2[nt], q, gw);
                            }
                        }
#pragma unroll
                        for (int ss = 0; ss < Cfg::KD / 32; ++ss)
                            if (ss == s)
#pragma unroll
                                for (int nt = 0; nt < Cfg::NT; ++nt)
#pragma unroll
                                    for (int e = 0; e < 4; ++e)
                                        part = __builtin_fmaf(S[ss][u][nt][e], o2[nt][e],
                                                              __builtin_fmaf(D[ss][u][nt][e], o1[nt][e], part));
                    }
                }
            }
            sum += (double)part;
            // (S, D) after these rows
            const int len = to - a;
            const Carry cy = len == Cfg::C ? full : carry_of(rate, (double)len);
#pragma unroll
            for (int s = 0; s < Cfg::KD / 32; ++s)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int nt = 0; nt < Cfg::NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            D[s][u][nt][e] = __builtin_fmaf((float)len, S[s][u][nt][e], D[s][u][nt][e]);
            carry_state<Cfg>(D, cy, mw != 0);
            carry_state<Cfg>(S, cy, mw != 0);
#pragma unroll
            for (int tb = 0; tb < Cfg::C / 32; ++tb) {
                bf16x8 z[Cfg::NT][Cfg::NP], zw[Cfg::NT][3];
#pragma unroll
                for (int nt = 0; nt < Cfg::NT; ++nt) {
                    col_frag<Cfg, Cfg::LDV>(z[nt], sV, tb, state_col_addr<Cfg>(nt, L), L);
                    weigh<Cfg>(zw[nt], z[nt], sW[0], tb, L);
                }
                state_add<Cfg>(S, sK, zw, tb, L);
#pragma unroll
                for (int nt = 0; nt < Cfg::NT; ++nt) weigh<Cfg>(zw[nt], z[nt], sW[1], tb, L);
                state_add<Cfg>(D, sK, zw, tb, L);
            }
            a = to;
        } while (a < n);
    }
    if (p.grad_state && seg == p.nseg - 1) {
        State<Cfg> G;
        load_state<Cfg>(G, p.grad_state + bh * words, vd, 1, kd, vd, L);
#pragma unroll
        for (int s = 0; s < Cfg::KD / 32; ++s)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int nt = 0; nt < Cfg::NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum += (double)D[s][u][nt][e] * (double)G[s][u][nt][e];
    }
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x, 64);
    if (L.lane == 0) sSum[L.w] = sum;
    __syncthreads();
    if (L.tid == 0) p.part[bh * p.nseg + seg] = (sSum[0] + sSum[1]) + (sSum[2] + sSum[3]);
}

__global__ __launch_bounds__(256) void ret_alpha_kernel(const double* part, const float* alpha, float* out, int64_t B,
                                                        int32_t H, int32_t nseg) {
    __shared__ double sSum[4];
    const int64_t h = blockIdx.x, n = B * nseg;
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 256) sum += part[((i / nseg) * H + h) * nseg + i % nseg];
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x, 64);
    if ((threadIdx.x & 63) == 0) sSum[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        const float a = alpha[h];
        const double s = (sSum[0] + sSum[1]) + (sSum[2] + sSum[3]);
        out[h] = a > 0.0f ? (float)-s : a < 0.0f ? (float)s : a == 0.0f ? 0.0f : a;     // NaN stays NaN
    }
}

// ------------------------------------------------------ gradients of shared heads
template <int NP>
__global__ __launch_bounds__(256) void ret_share_kernel(const float* part, void* out, int64_t units, int32_t heads,
                                                        int32_t G, int32_t d4) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < units; i += (int64_t)gridDim.x * 256) {
        const int64_t rk = i / d4, c = i % d4;             // (row, key head), four columns
        const f32x4* const x = (const f32x4*)part + rk * G * d4 + c;
        f32x4 s = x[0];
        for (int g = 1; g < G; ++g) s += x[(int64_t)g * d4];
        if (NP == 1) ((u32x2*)out)[i] = u32x2{f32x2_to_bf16x2(s[0], s[1]), f32x2_to_bf16x2(s[2], s[3])};
        else ((f32x4*)out)[i] = s;
    }
}

// ------------------------------------------------------------------- launches
namespace {
// f(Cfg) for the smallest tile that holds the state's kd rows and vd columns
template <int NP, class F>
void with_tiles(int kd, int vd, F&& f) {
    if (kd <= 64) {
        if (vd <= 64) f(RetCfg<NP, 64, 1>{});
        else f(RetCfg<NP, 64, 2>{});
    } else {
        if (vd <= 64) f(RetCfg<NP, 128, 1>{});
        else f(RetCfg<NP, 128, 2>{});
    }
}
template <class F>
void with_cfg(int planes, int kd, int vd, F&& f) {
    if (planes == 1) with_tiles<1>(kd, vd, f);
    else with_tiles<3>(kd, vd, f);
}
}  // namespace

hipError_t ret_walk_launch(int planes, const RetWalkArgs& a, int64_t B, hipStream_t s) {
    const dim3 grid((unsigned)a.nseg, (unsigned)a.H, (unsigned)B), block(256);
    with_cfg(planes, a.x.d, a.z.d, [&](auto cfg) {
        hipLaunchKernelGGL((ret_walk_kernel<decltype(cfg)>), grid, block, 0, s, a);
    });
    return hipGetLastError();
}

hipError_t ret_summary_launch(int planes, const RetSummaryArgs& a, int64_t B, hipStream_t s) {
    const dim3 grid((unsigned)(a.nseg - 1), (unsigned)a.H, (unsigned)B), block(256);
    with_cfg(planes, a.y.d, a.z.d, [&](auto cfg) {
        using Cfg = decltype(cfg);
        if (a.dstates) hipLaunchKernelGGL((ret_summary_kernel<Cfg, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((ret_summary_kernel<Cfg, false>), grid, block, 0, s, a);
    });
    return hipGetLastError();
}

hipError_t ret_state_scan_launch(const RetStateScanArgs& a, int64_t B, hipStream_t s) {
    const dim3 grid((unsigned)((a.words + 255) / 256), (unsigned)a.H, (unsigned)B), block(256);
    if (a.dstates) hipLaunchKernelGGL((ret_state_scan_kernel<true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((ret_state_scan_kernel<false>), grid, block, 0, s, a);
    return hipGetLastError();
}

hipError_t ret_sens_launch(int planes, const RetSensArgs& a, int64_t B, hipStream_t s) {
    const dim3 grid((unsigned)a.nseg, (unsigned)a.H, (unsigned)B), block(256);
    with_cfg(planes, a.q.d, a.v.d, [&](auto cfg) {
        hipLaunchKernelGGL((ret_sens_kernel<decltype(cfg)>), grid, block, 0, s, a);
    });
    return hipGetLastError();
}

hipError_t ret_alpha_launch(const double* part, const float* alpha, float* out, int64_t B, int32_t H, int32_t nseg,
                            hipStream_t s) {
    hipLaunchKernelGGL(ret_alpha_kernel, dim3((unsigned)H), dim3(256), 0, s, part, alpha, out, B, H, nseg);
    return hipGetLastError();
}

hipError_t ret_share_launch(int planes, const float* part, void* out, int64_t rows, int32_t heads, int32_t G, int32_t d,
                            hipStream_t s) {
    const int64_t units = rows * heads * (d / 4);
    const int64_t blocks = (units + 255) / 256 < 8192 ? (units + 255) / 256 : 8192;
    const dim3 grid((unsigned)blocks), block(256);
    if (planes == 1) hipLaunchKernelGGL((ret_share_kernel<1>), grid, block, 0, s, part, out, units, heads, G, d / 4);
    else hipLaunchKernelGGL((ret_share_kernel<3>), grid, block, 0, s, part, out, units, heads, G, d / 4);
    return hipGetLastError();
}

}  // namespace memoroid
