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
// decay in float and goes into the state as three planes, exactly, whether a state
// comes out or not: results do not depend on what else is asked for (two planes
// where none does: 975 us instead of 1022, 8 tapes of 4096, 16 heads of 128, forward
// and gradient).  With bf16 inputs P and the S that a row is multiplied with are
// operands of two planes, 2^-17 of a term, and the result is rounded to bf16 once,
// when it leaves: its error against 64 bits is the rounding's, 1.66e-3 (2.35e-3 with
// one plane each: 423 us instead of 459, T = 65536, 16 heads of 128).
//
// A value that is not finite must not reach other episodes, nor earlier rows of
// its own, through a zero of P or of the decays (0 * NaN): a chunk that holds one
// is walked row by row, by the recurrence itself in floats.
#include "retention_common.hpp"

namespace memoroid {

__device__ __forceinline__ void ret_header(WsHeader* hdr, uint64_t sig) {
    if (hdr && blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x < 16) {
        const u32x4 ones = {kEmpty32, kEmpty32, kEmpty32, kEmpty32};
        const u32x4 head = {kEmpty32, kEmpty32, (uint32_t)sig, (uint32_t)(sig >> 32)};
        ((u32x4*)hdr)[threadIdx.x] = threadIdx.x == 0 ? head : ones;
    }
}

// a role as head h of tape b sees it
struct Head {
    const void* p;
    int64_t row_bytes;
    int d;
};
template <class Cfg>
__device__ __forceinline__ Head head_of(const RetRole& x, int64_t b, int64_t h, int64_t T) {
    return Head{(const char*)x.p + (b * T * x.heads + h / x.share) * x.d * Cfg::ES, (int64_t)x.heads * x.d * Cfg::ES, x.d};
}
template <class Cfg>
__device__ __forceinline__ RetRows rows_of(const Head& x, int t0, int n, bool rev = false) {
    return ret_rows(x.p, x.row_bytes, x.d, Cfg::ES, t0, n, rev);
}
// A workgroup's run of chunks: steps r0 .. r1 - 1, in chunks of C from r0 on or,
// backwards, from r1 - 1 on; the last of them may be short.
template <class Cfg>
struct Run {
    int r0, r1, nch, rev;
    __device__ Run(int seg, int chunks, int T, int rev_) : r0(seg * chunks * Cfg::C), rev(rev_) {
        const int all = chunks * Cfg::C;
        r1 = T - r0 < all ? T : r0 + all;
        nch = (r1 - r0 + Cfg::C - 1) / Cfg::C;
    }
    __device__ __forceinline__ int rows(int ch) const {    // none past the run
        const int left = ch < nch ? r1 - r0 - ch * Cfg::C : 0;
        return left < Cfg::C ? left : Cfg::C;
    }
    __device__ __forceinline__ int first(int ch) const {   // the chunk's first step
        return ch >= nch ? r0 : rev ? r1 - ch * Cfg::C - rows(ch) : r0 + ch * Cfg::C;
    }
};

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
// tile `idx` of the triangle: rows 16 jb.. of y against rows 16 ib.. of x
__device__ __forceinline__ void tile_of(int idx, int& jb, int& ib) {
    ib = idx >= 6 ? 3 : idx >= 3 ? 2 : idx >= 1 ? 1 : 0;
    jb = idx - ib * (ib + 1) / 2;
}
template <class Cfg, int D>
__device__ __forceinline__ f32x4 pair_products(const uint16_t* sY, const uint16_t* sX, int jb, int ib, const RetLane& L) {
    f32x4 d = zero4();
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
        bf16x8 y[Cfg::NP], x[Cfg::NP];
        row_frag<Cfg, D>(y, sY, 16 * jb, s, L);
        row_frag<Cfg, D>(x, sX, 16 * ib, s, L);
        mma<Cfg::NP, Cfg::NP>(d, y, x);
    }
    return d;
}

// ---------------------------------------------------------------- summaries
// What a segment adds to the state after it: the sum over its rows from the last
// begin on.  Reads y and z once: T = 65536, 16 heads of 128, bf16, 136 us, 4.1 TB/s
// with the states written (8 tapes of 4096: 63 us, 3.6 TB/s); its wavefronts wait
// for 0.35 of their time.
template <class Cfg>
__global__ __launch_bounds__(Cfg::THREADS, 4) void ret_summary_kernel(RetSummaryArgs p) {
    __shared__ __attribute__((aligned(16))) uint16_t sY[Cfg::NP * Cfg::C * Cfg::KD];
    __shared__ __attribute__((aligned(16))) uint16_t sZ[Cfg::NP * Cfg::C * Cfg::VD];
    __shared__ Powers<Cfg::C + 1> sPw;
    __shared__ __attribute__((aligned(16))) float sW[Cfg::C];
    RetLane L;
    const int64_t seg = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    ret_header(p.hdr, p.sig);
    const double rate = fabs((double)p.alpha[h]);
    sPw.fill(rate, L.tid);
    const Head hy = head_of<Cfg>(p.y, b, h, p.T), hz = head_of<Cfg>(p.z, b, h, p.T);
    const uint8_t* const start = p.start + b * p.T;
    const Run<Cfg> run((int)seg, p.chunks, (int)p.T, 0);  // a whole segment: the last has no summary
    State<Cfg> S;
    zero_state<Cfg>(S);
    Owed owed;
    __syncthreads();                                       // the powers are there
    bool any = false;
    RetTile<Cfg, Cfg::KD> ty;
    RetTile<Cfg, Cfg::VD> tz;
    uint32_t flag;
    auto fetch = [&](int ch) {
        const int t0 = run.first(ch), n = run.rows(ch);
        flag = ret_flag(start, t0, n, (int)p.T, false, L.lane);
        ty.fetch(rows_of<Cfg>(hy, t0, n), L);
        tz.fetch(rows_of<Cfg>(hz, t0, n), L);
    };
    fetch(0);
#pragma unroll 1
    for (int ch = 0; ch < run.nch; ++ch) {
        L.again();
        const uint64_t m = __ballot(flag != 0u);
        const int from = m ? last_begin(m) : 0;
        any = any || m != 0;
        bool take = false;
        if (m) owed.none();
        else take = owed.add(sPw, Cfg::C);
        const Carry cy = carry_by(owed.now);
        if (take) owed.none();
        if (m) {
            ty.keep(from, Cfg::C, L);
            tz.keep(from, Cfg::C, L);
        }
        barrier_lds();                                     // the last chunk's operands have been read
        ty.stage(sY, L);
        tz.stage(sZ, L);
        if (L.tid < Cfg::C)
            sW[L.tid] = L.tid >= from ? sPw.f(Cfg::C - 1 - L.tid) * (float)owed.inverse : 0.0f;
        fetch(ch + 1);
        barrier_lds();
        settle<Cfg>(S, m != 0, take, cy);
#pragma unroll
        for (int tb = 0; tb < Cfg::C / 32; ++tb) {
            bf16x8 z[Cfg::NP], zw[3];
            col_frag<Cfg, Cfg::VD>(z, sZ, tb, state_col_addr(L), L);
            weigh<Cfg>(zw, z, sW, tb, L);
#pragma unroll
            for (int s = 0; s < Cfg::KS; ++s)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    bf16x8 y[Cfg::NP];
                    col_frag<Cfg, Cfg::KD>(y, sY, tb, state_row_addr(s, u, L), L);
                    mma<Cfg::NP, 3>(S[s][u], y, zw);
                }
        }
    }
    L.again();
    const int64_t words = (int64_t)p.y.d * p.z.d;
    store_state<Cfg>(S, p.states + ((b * p.H + h) * p.nseg + seg) * words, p.z.d, 1, p.y.d, p.z.d, (float)owed.now, false, L);
    if (h == 0 && L.tid == 0) p.R[b * p.nseg + seg] = any ? kSegBegins : 0;
}

// ------------------------------------------- what the gradient needs of a segment
// With f_t = scale gamma^(t - r0) for the steps t of a segment that no begin
// separates from its first step r0,
//     S  = what the segment adds to the state after it,
//     U  = sum f_t q_t^T g_t, what it adds to the gradient of the state at r0,
// and for the gradient of the rates (ALPHA)
//     D  = dS / dlog gamma,   E = sum (t - r0) f_t q_t^T g_t,
//     part = the segment's own share of dL/dlog gamma, as if the state before it
//            were zero.
// With D_t = dS_t / dlog gamma = gamma (D_{t-1} + S_{t-1}) + 0 inside an episode,
//     dL/dlog gamma = scale sum_t q_t D_t g_t^T   (+ D_{T-1} . grad_state),
// which per chunk, (S, D) before it, o1 = sum gamma^i q_i^T g_i and o2 = sum i gamma^i
// q_i^T g_i over its rows whose episode began earlier, is
//     sum_ij (i-j) gamma^(i-j) (q_i . k_j)(g_i . v_j)  +  gamma (S . (o1 + o2) + D . o1).
// The outer products arrive in the state's own layout, so they meet S and D as
// floats in registers, and the pairs' products are not rounded either: nothing of
// dL/dlog gamma is rounded to bf16.  What a state before the segment adds to it,
// gamma (S . (U + E) + D . U), follows in the state scan.
//
// One pass reads q, k, v and g once, with the states in registers, 64 rows of each per
// wavefront (RetCfg64).  With four states of 128 x 128 a workgroup of 16 wavefronts
// takes all 128 registers of each and spills 16; what the next chunk's rows need of
// them is free only behind the outer products, so they are fetched there.  T = 4096, 8
// tapes, 16 heads, bf16: 326 us.  Its VALU instructions take about 210 of those, the
// matrix cores 86; half of them form the rows' weights in three planes, once for each
// 64 of the state's rows.  In short runs, before the clocks have risen, 380 us: 504
// with the rows fetched before the products, 487 in two passes of eight wavefronts with
// two states each, 531 with the weights formed once for all rows (the second state's
// columns in lanes c >= 8 of a wavefront with 8 columns), since more registers spill.
//
// A value that is not finite would reach other episodes and earlier rows through
// zero weights.  Without ALPHA the rows that take no part become zeros.  With
// ALPHA, where every row takes part in something, the segment is done again row by
// row.

// The sums of ret_prep_kernel, with ALPHA, of a segment that holds a value that is not
// finite, by the recurrences themselves in floats.  Returns this lane's part.
template <class Cfg>
__device__ __forceinline__ double prep_rows(const RetPrepArgs& p, const Run<Cfg>& run, const Head& hq, const Head& hk,
                                            const Head& hv, const Head& hg, const uint8_t* start, double rate,
                                            uint16_t* sQ, uint16_t* sK, uint16_t* sV, uint16_t* sG, State<Cfg>& S,
                                            State<Cfg>& D, State<Cfg>& U, State<Cfg>& E, const RetLane& L) {
    const Carry one = carry_of(rate, 1.0);
    zero_state<Cfg>(S);
    zero_state<Cfg>(D);
    zero_state<Cfg>(U);
    zero_state<Cfg>(E);
    bool open = true;
    double sum = 0.0;
#pragma unroll 1
    for (int ch = 0; ch < run.nch; ++ch) {
        RetTile<Cfg, Cfg::KD> tq, tk;
        RetTile<Cfg, Cfg::VD> tv, tg;
        const int t0 = run.first(ch), n = run.rows(ch);
        const uint64_t m = __ballot(ret_flag(start, t0, n, (int)p.T, false, L.lane) != 0u);
        tq.fetch(rows_of<Cfg>(hq, t0, n), L);
        tk.fetch(rows_of<Cfg>(hk, t0, n), L);
        tv.fetch(rows_of<Cfg>(hv, t0, n), L);
        tg.fetch(rows_of<Cfg>(hg, t0, n), L);
        __syncthreads();
        tq.stage(sQ, L);
        tk.stage(sK, L);
        tv.stage(sV, L);
        tg.stage(sG, L);
        __syncthreads();
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
            const int t = ch * Cfg::C + i;                 // steps since r0
            const bool begin = (m >> i) & 1ull;
            open = open && !(begin && t > 0);
            const float f = decay_pow(rate, (double)t) * p.scale;
            const float v = tile_value<Cfg, Cfg::VD>(sV, i, state_col(L));
            const float g = tile_value<Cfg, Cfg::VD>(sG, i, state_col(L));
            float dot = 0.0f;
#pragma unroll
            for (int s = 0; s < Cfg::KS; ++s) {
                float q[8], k[8];
                row_values<Cfg, Cfg::KD>(q, sQ, i, s, L);
                row_values<Cfg, Cfg::KD>(k, sK, i, s, L);
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const int u = x >> 2, e = x & 3;
                    const float d = begin ? 0.0f : one(D[s][u][e] + S[s][u][e]);
                    D[s][u][e] = d;
                    S[s][u][e] = __builtin_fmaf(k[x], v, begin ? 0.0f : one(S[s][u][e]));
                    dot = __builtin_fmaf(q[x], d, dot);
                    const float o = q[x] * (f * g);
                    U[s][u][e] = open ? U[s][u][e] + o : U[s][u][e];
                    E[s][u][e] = open && t > 0 ? __builtin_fmaf((float)t, o, E[s][u][e]) : E[s][u][e];
                }
            }
            if (!begin && t > 0) sum += (double)(dot * p.scale * g);
        }
    }
    return sum;
}

template <class Cfg, bool ALPHA>
__global__ __launch_bounds__(Cfg::THREADS, Cfg::THREADS == 1024 ? 4 : 2) void ret_prep_kernel(RetPrepArgs p) {
    // four states in 128 registers: nothing is read ahead of its use
    constexpr bool kFull = Cfg::THREADS == 1024 && ALPHA;
    __shared__ __attribute__((aligned(16))) uint16_t sQ[Cfg::NP * Cfg::C * Cfg::KD];
    __shared__ __attribute__((aligned(16))) uint16_t sK[Cfg::NP * Cfg::C * Cfg::KD];
    __shared__ __attribute__((aligned(16))) uint16_t sV[Cfg::NP * Cfg::C * Cfg::VD];
    __shared__ __attribute__((aligned(16))) uint16_t sG[Cfg::NP * Cfg::C * Cfg::VD];
    __shared__ Powers<Cfg::C + 1> sPw;
    __shared__ float sAge[Cfg::C + 16];                    // [16 + n]: n gamma^n scale, 0 for n < 0
    __shared__ __attribute__((aligned(16))) float sW[4][Cfg::C];
    __shared__ double sSum[Cfg::W];
    RetLane L;
    const int wave = L.w;
    L.k0 = wave / Cfg::CW * 64;
    L.w = wave % Cfg::CW;
    const int64_t seg = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    ret_header(p.hdr, p.sig);
    const double rate = fabs((double)p.alpha[h]);
    sPw.fill(rate, L.tid);
    if (ALPHA && L.tid < Cfg::C + 16) {
        const int age = L.tid - 16;
        sAge[L.tid] = age < 0 ? 0.0f : decay_pow(rate, age) * (float)age * p.scale;
    }
    const int kd = p.q.d, vd = p.v.d;
    const Head hq = head_of<Cfg>(p.q, b, h, p.T), hk = head_of<Cfg>(p.k, b, h, p.T), hv = head_of<Cfg>(p.v, b, h, p.T),
               hg = head_of<Cfg>(p.g, b, h, p.T);
    const uint8_t* const start = p.start + b * p.T;
    const Run<Cfg> run((int)seg, p.chunks, (int)p.T, 0);

    RetTile<Cfg, Cfg::KD> tq, tk;
    RetTile<Cfg, Cfg::VD> tv, tg;
    uint32_t flag;
    auto fetch = [&](int ch) {
        const int t0 = run.first(ch), n = run.rows(ch);
        flag = ret_flag(start, t0, n, (int)p.T, false, L.lane);
        tq.fetch(rows_of<Cfg>(hq, t0, n), L);
        tk.fetch(rows_of<Cfg>(hk, t0, n), L);
        tv.fetch(rows_of<Cfg>(hv, t0, n), L);
        tg.fetch(rows_of<Cfg>(hg, t0, n), L);
    };
    fetch(0);
    State<Cfg> S, D, U, E;
    zero_state<Cfg>(S);
    zero_state<Cfg>(U);
    if (ALPHA) {
        zero_state<Cfg>(D);
        zero_state<Cfg>(E);
    }
    Owed owed;
    __syncthreads();                                       // the powers are there
    const float gamma = uniform(sPw.f(1));
    double sum = 0.0, reach = 1.0;                         // gamma^(steps before the rows at hand)
    bool open = true;                                      // no begin since r0
    uint32_t begins = 0, bad = 0;
#pragma unroll 1
    for (int ch = 0; ch < run.nch; ++ch) {
        L.again();
        const int n = run.rows(ch);
        const uint64_t m = __ballot(flag != 0u);
        if (ch == 0 && (m & 1ull)) begins |= kSegBeginsFirst;
        if (ALPHA) bad |= tq.bad() | tk.bad() | tv.bad() | tg.bad();
        const uint64_t mo = ch == 0 ? m & ~1ull : m;   // a begin at r0 separates nothing from it
        if (m) begins |= kSegBegins;
        if (mo) begins |= kSegBeginsBack;
        // rows from `from` on enter S, rows before `to` go on from before the chunk
        const int from = m ? last_begin(m) : 0, to = mo ? __builtin_ctzll(mo) : n;
        const float was = uniform((float)owed.now);
        bool take = false;
        if (m) owed.none();
        else take = owed.add(sPw, n);
        const Carry cy = carry_by(owed.now);
        if (take) owed.none();
        const float far = uniform((float)reach), off = (float)(ch * Cfg::C);
        if (!ALPHA && m) {
            tk.keep(from, Cfg::C, L);
            tv.keep(from, Cfg::C, L);
            tq.keep(0, open ? to : 0, L);
            tg.keep(0, open ? to : 0, L);
        }
        barrier_lds();                                 // the last operands have been read
        tq.stage(sQ, L);
        tk.stage(sK, L);
        tv.stage(sV, L);
        tg.stage(sG, L);
        if (L.tid < Cfg::C) {
            const int i = L.tid;
            const float w = i >= from && i < n ? sPw.f(i < n ? n - 1 - i : 0) * (float)owed.inverse : 0.0f;
            sW[0][i] = w;
            const float f = i < to ? sPw.f(i) * p.scale : 0.0f;
            sW[2][i] = f;
            if (ALPHA) {
                sW[1][i] = w * (float)(n - 1 - i);
                sW[3][i] = f * (float)i;
            }
        }
        barrier_lds();
        if constexpr (ALPHA) {
            float part = 0.0f;
#pragma unroll
            for (int i = 0; i < (Cfg::NTILE + Cfg::W - 1) / Cfg::W; ++i) {
                const int idx = Cfg::W * i + wave;
                if (idx >= Cfg::NTILE) break;
                int jb, ib;
                tile_of(idx, jb, ib);
                const f32x4 x = pair_products<Cfg, Cfg::KD>(sK, sQ, jb, ib, L);
                const f32x4 y = pair_products<Cfg, Cfg::VD>(sV, sG, jb, ib, L);
                const int row = 16 * ib + L.c, age = row - 16 * jb - 4 * L.g;
                const uint64_t mr = m & upto(row);
                const int oldest = mr ? row - last_begin(mr) : row;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    part += age - r > 0 && age - r <= oldest ? x[r] * y[r] * sAge[age - r + 16] : 0.0f;
            }
            sum += (double)part;
        }
        // ---- rows of the first episode: outer products of q and g.  Without any
        // such row nothing is touched, so that values of S that are not finite
        // stay out
        if (to > 0 && (ALPHA || open)) {
            const float use = open ? far : 0.0f;
            float part = 0.0f;
            // o1, then o2: one set of weighted g at a time, for the registers
#pragma unroll
            for (int k = 0; k < (ALPHA ? 2 : 1); ++k) {
                bf16x8 gw[Cfg::C / 32][3];
#pragma unroll
                for (int tb = 0; tb < Cfg::C / 32; ++tb) {
                    bf16x8 g[Cfg::NP];
                    col_frag<Cfg, Cfg::VD>(g, sG, tb, state_col_addr(L), L);
                    weigh<Cfg>(gw[tb], g, sW[2 + k], tb, L);
                }
#pragma unroll
                for (int s = 0; s < Cfg::KS; ++s)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        f32x4 o = zero4();
#pragma unroll
                        for (int tb = 0; tb < Cfg::C / 32; ++tb) {
                            bf16x8 q[Cfg::NP];
                            col_frag<Cfg, Cfg::KD>(q, sQ, tb, state_row_addr(s, u, L), L);
                            mma<Cfg::NP, 3>(o, q, gw[tb]);
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (k == 0) U[s][u][e] = __builtin_fmaf(use, o[e], U[s][u][e]);
                            if (ALPHA) E[s][u][e] = __builtin_fmaf(k == 0 ? use * off : use, o[e], E[s][u][e]);
                            if (ALPHA)
                                part = __builtin_fmaf(k == 0 ? S[s][u][e] + D[s][u][e] : S[s][u][e], o[e], part);
                        }
                        if constexpr (kFull) __builtin_amdgcn_sched_barrier(0);
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
            // (before the first step there is no state, and no state is NaN)
            if (ALPHA && ch > 0) sum += (double)(part * (was * gamma));
        }
        fetch(ch + 1);                                 // here, for the registers
        // ---- (S, D) after the rows
        if constexpr (ALPHA) {
            const float steps = (float)n;
            each<Cfg>(D, [&](float x, int s, int u, int e) { return __builtin_fmaf(steps, S[s][u][e], x); });
            settle<Cfg>(D, m != 0, take, cy);
        }
        settle<Cfg>(S, m != 0, take, cy);
#pragma unroll
        for (int tb = 0; tb < Cfg::C / 32; ++tb) {
            bf16x8 z[Cfg::NP];
            col_frag<Cfg, Cfg::VD>(z, sV, tb, state_col_addr(L), L);
#pragma unroll
            for (int k = 0; k < (ALPHA ? 2 : 1); ++k) {
                bf16x8 zw[3];
                weigh<Cfg>(zw, z, sW[k], tb, L);
#pragma unroll
                for (int s = 0; s < Cfg::KS; ++s)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        bf16x8 y[Cfg::NP];
                        col_frag<Cfg, Cfg::KD>(y, sK, tb, state_row_addr(s, u, L), L);
                        mma<Cfg::NP, 3>(k ? D[s][u] : S[s][u], y, zw);
                        if constexpr (kFull) __builtin_amdgcn_sched_barrier(0);
                    }
            }
        }
        open = open && mo == 0;
        reach = uniform(reach * sPw.of[n]);
    }
    L.again();
    const int64_t words = (int64_t)kd * vd, bh = b * p.H + h, at = (bh * p.nseg + seg) * words;
    float now = (float)owed.now;
    if constexpr (ALPHA) {
        // a value that is not finite, in the inputs or by overflow
        if (__syncthreads_or(bad != 0u || !(fabs(sum) < (double)__builtin_inff()))) {
            sum = prep_rows<Cfg>(p, run, hq, hk, hv, hg, start, rate, sQ, sK, sV, sG, S, D, U, E, L);
            now = 1.0f;
        }
    }
    store_state<Cfg>(S, p.states + at, vd, 1, kd, vd, now, false, L);
    store_state<Cfg>(U, p.rstates + at, vd, 1, kd, vd, 1.0f, false, L);
    if (ALPHA) store_state<Cfg>(D, p.dstates + at, vd, 1, kd, vd, now, false, L);
    if (ALPHA) store_state<Cfg>(E, p.estates + at, vd, 1, kd, vd, 1.0f, false, L);
    if (ALPHA) {
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x, 64);
        if (L.lane == 0) sSum[wave] = sum;
        __syncthreads();
        if (L.tid == 0) {
            double s = 0.0;
#pragma unroll
            for (int i = 0; i < Cfg::W; ++i) s += sSum[i];
            p.part[bh * p.nparts + seg] = s;
        }
    }
    if (h == 0 && L.tid == 0) {
        if (run.r1 < p.T && start[run.r1] != 0) begins |= kSegBeginsBack;
        p.R[b * p.nseg + seg] = (uint8_t)begins;
    }
}

// ---------------------------------------------------------------- state scan
// out[i] is the state after segment i: its summary, plus gamma^rows times
// the state before it where it holds no begin step; with DOT the derivative
// likewise, d' = own + gamma^rows (d + rows s).  GROUPS threads share a 16-byte
// column of the states, each with RPT consecutive segments of it in registers, all
// loads in flight at once; the groups combine through LDS.  One read and one write
// of the states.  One group where there are few segments or many columns (3
// segments of 128 heads of 128 x 128: 10 us, 294 us in 32 groups; 31 segments of 16
// such heads: 12 us, 53 in 32 groups in a short run, in which one takes 16), else 32
// (128 segments of 4 heads of 64 x 64: 9 us, 39 us one segment after the other).
template <bool DOT>
struct SegState {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f}, d = {0.0f, 0.0f, 0.0f, 0.0f};
    // this after `own`, a run that decays by cy over `rows` steps
    __device__ __forceinline__ void then(const f32x4& os, const f32x4& od, bool begins, Carry cy, float rows) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (DOT) d[e] = begins ? od[e] : od[e] + cy(__builtin_fmaf(rows, s[e], d[e]));
            s[e] = begins ? os[e] : os[e] + cy(s[e]);
        }
    }
};

template <int GROUPS, int RPT, bool DOT>
__device__ __forceinline__ void state_scan_body(const RetStateScanArgs& p, int64_t b) {
    constexpr int kCols = 256 / GROUPS, kTile = GROUPS * RPT;
    __shared__ f32x4 sTot[GROUPS > 1 && DOT ? 2 : 1][GROUPS][GROUPS > 1 ? kCols : 1];
    __shared__ uint32_t sFlag[GROUPS];
    __shared__ double sSum[DOT ? 4 : 1];
    const int col = threadIdx.x % kCols, grp = threadIdx.x / kCols;
    const int64_t h = blockIdx.y, bh = b * p.H + h;
    const int c4 = (int)blockIdx.x * kCols + col, w4 = p.words / 4;   // words is a multiple of 64
    const bool in = c4 < w4;
    const double rate = fabs((double)p.alpha[h]), rows = (double)p.rows, last = (double)p.last_rows;
    // the nseg - 1 segments that have one behind them in scan order; with DOT the
    // last one too, for what it takes from the state before it
    const int n = DOT ? p.nseg : p.nseg - 1;
    const Carry one = carry_of(rate, rows), many = carry_of(rate, rows * RPT);
    // Backwards the last segment, which may be short, comes first, and the seed
    // belongs to its last step itself: one decay less.
    const Carry one0 = p.rev ? carry_of(rate, last - 1.0) : one;
    const Carry many0 = p.rev ? carry_of(rate, last - 1.0 + rows * (RPT - 1)) : many;
    const Carry one_last = carry_of(rate, last);
    const uint32_t bit = p.rev ? kSegBeginsBack : kSegBegins;
    const f32x4* const S = (const f32x4*)p.states + bh * p.nseg * w4 + c4;
    f32x4* const O = (f32x4*)p.out + bh * p.nseg * w4 + c4;
    f32x4* const D = DOT ? (f32x4*)p.dstates + bh * p.nseg * w4 + c4 : nullptr;
    const f32x4* const U = DOT ? (const f32x4*)p.rstates + bh * p.nseg * w4 + c4 : nullptr;
    const f32x4* const E = DOT ? (const f32x4*)p.estates + bh * p.nseg * w4 + c4 : nullptr;
    const uint8_t* const R = p.R + b * p.nseg;
    auto seg_of = [&](int l) { return p.rev ? p.nseg - 1 - l : l; };
    const f32x4 zero = zero4();
    double sum = 0.0;
    SegState<DOT> before;                                  // the state before the tile
    if (p.seed && in) before.s = ((const f32x4*)p.seed)[bh * w4 + c4];
    for (int base = 0; base < n; base += kTile) {
        f32x4 x[RPT], y[DOT ? RPT : 1];
        uint32_t fl[RPT];
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int l = base + grp * RPT + i, sg = seg_of(l);
            const bool have = in && l < n;
            x[i] = have ? S[(int64_t)sg * w4] : zero;
            if (DOT) y[DOT ? i : 0] = have ? D[(int64_t)sg * w4] : zero;
            fl[i] = l < n ? R[l < n ? sg : 0] : 0u;
        }
        SegState<DOT> mine = before;                       // the state before this thread's run
        if constexpr (GROUPS > 1) {
            SegState<DOT> tot;
            bool any = false;
#pragma unroll
            for (int i = 0; i < RPT; ++i) {
                tot.then(x[i], y[DOT ? i : 0], (fl[i] & bit) != 0u, one, (float)p.rows);
                any |= (fl[i] & bit) != 0u;
            }
            __syncthreads();                               // the last tile's totals have been read
            sTot[0][grp][col] = tot.s;
            if (DOT) sTot[DOT ? 1 : 0][grp][col] = tot.d;
            if (col == 0) sFlag[grp] = any;
            __syncthreads();
#pragma unroll 4
            for (int k = 0; k < GROUPS; ++k) {
                if (k == grp) mine = before;
                before.then(sTot[0][k][col], sTot[DOT ? 1 : 0][k][col], sFlag[k] != 0u, base == 0 && k == 0 ? many0 : many,
                            (float)p.rows * RPT);
            }
        }
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int l = base + grp * RPT + i;
            const bool have = in && l < n;
            if constexpr (DOT) {
                // gamma (S . (U + E) + D . U), where the segment's first step goes on
                if (have && !(fl[i] & kSegBeginsFirst)) {
                    const f32x4 u = U[(int64_t)l * w4], e = E[(int64_t)l * w4];
                    float d = 0.0f;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        d = __builtin_fmaf(mine.s[k], u[k] + e[k], __builtin_fmaf(mine.d[k], u[k], d));
                    sum += (double)(d * decay_pow(rate, 1.0));
                }
                const bool at_end = l == p.nseg - 1;
                mine.then(x[i], y[DOT ? i : 0], (fl[i] & bit) != 0u, at_end ? one_last : one,
                          (float)(at_end ? p.last_rows : p.rows));
                if (have && !at_end) {
                    O[(int64_t)l * w4] = mine.s;
                    D[(int64_t)l * w4] = mine.d;
                }
                if (have && at_end && p.grad_state) {      // D after the tape . grad_state
                    const f32x4 g = ((const f32x4*)p.grad_state)[bh * w4 + c4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) sum += (double)mine.d[k] * (double)g[k];
                }
            } else {
                mine.then(x[i], zero, (fl[i] & bit) != 0u, l == 0 ? one0 : one, 0.0f);
                if (have) O[(int64_t)seg_of(l) * w4] = mine.s;
            }
        }
        if constexpr (GROUPS == 1) before = mine;
    }
    if constexpr (DOT) {
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m, 64);
        if ((threadIdx.x & 63) == 0) sSum[threadIdx.x >> 6] = sum;
        __syncthreads();
        if (threadIdx.x == 0)
            p.part[bh * p.nparts + p.nseg + blockIdx.x] = (sSum[0] + sSum[1]) + (sSum[2] + sSum[3]);
    }
}

// tapes 0 .. B - 1 forwards, then (with a grid for them) backwards
template <int GROUPS, int RPT, bool DOT>
__global__ __launch_bounds__(256) void ret_state_scan_kernel(RetStateScanArgs p, RetStateScanArgs back, int B) {
    if ((int)blockIdx.z < B) state_scan_body<GROUPS, RPT, DOT>(p, blockIdx.z);
    else state_scan_body<GROUPS, RPT, false>(back, blockIdx.z - B);
}

// ------------------------------------------------------- gradient of the rates
// grad_alpha[h] = -sign(alpha_h) times the sum of the shares over tapes, in a fixed
// order
__device__ __forceinline__ void alpha_sum(const RetWalkSet& p, int64_t h) {
    __shared__ double sSum[16];
    const int threads = blockDim.x;
    const int64_t n = p.B * p.nparts;
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += threads) sum += p.part[((i / p.nparts) * p.H + h) * p.nparts + i % p.nparts];
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x, 64);
    if ((threadIdx.x & 63) == 0) sSum[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        const float a = p.w[0].alpha[h];
        double s = 0.0;
        for (int i = 0; i < threads / 64; ++i) s += sSum[i];
        p.grad_alpha[h] = a > 0.0f ? (float)-s : a < 0.0f ? (float)s : a == 0.0f ? 0.0f : a;   // NaN stays NaN
    }
}

// ---------------------------------------------------------------------- walk
// The masked, decayed products of a chunk's rows in tiles as operands of the next
// product, a tile or two per wavefront.  by_age[16 + n]: the weight of a partner n
// steps back, 0 for n < 0;  m: begin bits.  Returns whether a row's
// product with itself came out not finite: every x and y that is not finite shows
// there (and so does one that overflows).
template <class Cfg>
__device__ __forceinline__ bool pairs(u32x2 (&sP)[Cfg::NTILE][Cfg::FP][64], const uint16_t* sX, const uint16_t* sY,
                                      const float* by_age, uint64_t m, const RetLane& L) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < (Cfg::NTILE + Cfg::W - 1) / Cfg::W; ++i) {
        const int idx = Cfg::W * i + L.w;
        if (idx >= Cfg::NTILE) break;
        int jb, ib;
        tile_of(idx, jb, ib);
        f32x4 d = pair_products<Cfg, Cfg::KD>(sY, sX, jb, ib, L);
        const int row = 16 * ib + L.c, age = row - 16 * jb - 4 * L.g;      // of register 0
        if (ib == jb)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                bad |= age == r && !(fabsf(d[r]) < __builtin_inff());
                d[r] = age >= r ? d[r] : 0.0f;                             // (its weight is 0, the product may have overflowed)
            }
#pragma unroll
        for (int r = 0; r < 4; ++r) d[r] *= by_age[age - r + 16];
        if (m) {                                                           // age of the row's first partner
            const uint64_t mr = m & upto(row);
            const int oldest = mr ? row - last_begin(mr) : row;
#pragma unroll
            for (int r = 0; r < 4; ++r) d[r] = age - r <= oldest ? d[r] : 0.0f;
        }
        uint32_t lo[Cfg::FP], hi[Cfg::FP];
        planes2<Cfg::FP>(d[0], d[1], lo);
        planes2<Cfg::FP>(d[2], d[3], hi);
#pragma unroll
        for (int q = 0; q < Cfg::FP; ++q) sP[idx][q][L.lane] = u32x2{lo[q], hi[q]};
    }
    return bad;
}

// Two workgroups on a CU, whose phases (staging, pairs, rows against the state, rows
// into it) cover each other's waits.  T = 65536, 16 heads of 128, bf16: 303 us, 3.5
// TB/s of x, y, z and out; 8 tapes of 4096: 149 us, 3.6 TB/s, and 441 for the
// gradient's three walks, with the matrix cores busy for a quarter of the time and waits
// in 0.42 of the wavefronts'.  fp32, T = 32768, 4 heads of 64: 41 us, and 97 for three: 440
// TFLOP/s of bf16 products, six for one of floats, 0.38 of what a large bf16 product
// reaches.
template <class Cfg>
__global__ __launch_bounds__(Cfg::THREADS, Cfg::VD == 128 ? 4 : Cfg::KD == 128 ? 2 : 3)
    void ret_walk_kernel(RetWalkSet set) {
    // Tasks of the walks in turn, eight at a time: the workgroups of the same task
    // of two walks run on the same of the eight dies, one behind the other, and what
    // both read comes from its cache once.  Behind them, the rates' gradients.
    const int64_t id = blockIdx.x;
    if (id >= set.blocks) {
        alpha_sum(set, id - set.blocks);
        return;
    }
    const RetWalkArgs& p = set.w[(id >> 3) % set.n];
    const int64_t task = (id >> 3) / set.n * 8 + (id & 7);
    if (task >= set.tasks) return;
    __shared__ __attribute__((aligned(16))) uint16_t sX[Cfg::NP * Cfg::C * Cfg::KD];
    __shared__ __attribute__((aligned(16))) uint16_t sY[Cfg::NP * Cfg::C * Cfg::KD];
    __shared__ __attribute__((aligned(16))) uint16_t sZ[Cfg::NP * Cfg::C * Cfg::VD];
    // bf16 out: rows gathered here, so that they leave 16 bytes a lane, a row at a
    // time (a wavefront's own 32 bytes of a row doubled the bytes written)
    __shared__ __attribute__((aligned(16))) uint16_t sO[Cfg::NP == 1 ? Cfg::C * Cfg::VD : 8];
    __shared__ u32x2 sP[Cfg::NTILE][Cfg::FP][64];
    __shared__ Powers<Cfg::C + 1> sPw;
    __shared__ float sAge[Cfg::C + 16];
    __shared__ __attribute__((aligned(16))) float sW[Cfg::C];
    __shared__ uint32_t sBad[Cfg::W];
    RetLane L;
    const int64_t seg = task % p.nseg, h = task / p.nseg % p.H, b = task / p.nseg / p.H;
    if (id == 0) ret_header(p.hdr, p.sig);
    const double rate = fabs((double)p.alpha[h]);
    sPw.fill(rate, L.tid);
    if (L.tid < Cfg::C + 16) sAge[L.tid] = L.tid < 16 ? 0.0f : decay_pow(rate, L.tid - 16) * p.p_scale;
    const Head hx = head_of<Cfg>(p.x, b, h, p.T), hy = head_of<Cfg>(p.y, b, h, p.T), hz = head_of<Cfg>(p.z, b, h, p.T);
    const uint8_t* const start = p.start + b * p.T;
    const int64_t words = (int64_t)p.x.d * p.z.d, bh = b * p.H + h;
    const Run<Cfg> run((int)seg, p.chunks, (int)p.T, p.rev);
    const int64_t at_start = p.rev ? p.nseg - 1 : 0;       // the segment that the walk begins with
    const int os = Cfg::NP == 1 && !p.out_f32 ? 2 : 4;
    auto rows_out = [&](int ch) {
        return ret_rows((char*)p.out + (b * p.T * p.H + h) * p.z.d * os, (int64_t)p.H * p.z.d * os, p.z.d, os, run.first(ch),
                        run.rows(ch), p.rev);
    };

    RetTile<Cfg, Cfg::KD> tx, ty;
    RetTile<Cfg, Cfg::VD> tz;
    uint32_t flag;
    auto fetch = [&](int ch) {
        const int t0 = run.first(ch), n = run.rows(ch);
        flag = ret_flag(start, t0, n, (int)p.T, p.rev, L.lane);
        tx.fetch(rows_of<Cfg>(hx, t0, n, p.rev), L);
        ty.fetch(rows_of<Cfg>(hy, t0, n, p.rev), L);
    };
    auto fetch_z = [&](int ch) { tz.fetch(rows_of<Cfg>(hz, run.first(ch), run.rows(ch), p.rev), L); };
    Owed owed;
    __syncthreads();                                       // the powers are there
    bool held = false;                                     // the last chunk's rows wait in sO
    auto put_rows = [&](int ch) {
        const RetRows o = rows_out(ch);
        constexpr int UPR = Cfg::VD / 8, RS = Cfg::THREADS / UPR;
#pragma unroll
        for (int i = 0; i < Cfg::C / RS; ++i) {
            const int row = L.tid / UPR + i * RS, unit = L.tid % UPR;
            const u32x4 x = *(const u32x4*)(sO + row * Cfg::VD + swizzled<Cfg::VD>(unit, row) * 8);
            __builtin_amdgcn_raw_buffer_store_b128(x, o.r, (int)o.offset(row, 8 * unit, 2), 0, 0);
        }
    };
    fetch(0);
    fetch_z(0);
    State<Cfg> S;
    load_state<Cfg>(S, seg == at_start ? (p.seed ? p.seed + bh * words : nullptr)
                                       : p.states + (bh * p.nseg + (p.rev ? seg + 1 : seg - 1)) * words,
                    p.sk, p.sv, p.x.d, p.z.d, L);
#pragma unroll 1
    for (int ch = 0; ch < run.nch; ++ch) {
        L.again();
        const int n = run.rows(ch);
        const uint64_t m = __ballot(flag != 0u);
        const bool bad_z = tz.bad() != 0u;
        // the gradient of the state after the tape belongs to the last step
        const int e = p.rev && seg == at_start && ch == 0 ? 0 : 1;
        const float was = uniform((float)owed.now), before = was * p.inter_scale;
        bool take = false;
        if (m) owed.none();
        else take = owed.add(sPw, n - 1 + e);
        const Carry cy = carry_by(owed.now);
        if (take) owed.none();
        barrier_lds();                                     // the last chunk's operands have been read
        tx.stage(sX, L);
        ty.stage(sY, L);
        tz.stage(sZ, L);
        // weights of the rows into the state: no begin step after them
        if (L.tid < Cfg::C) {
            const int from = m ? last_begin(m) : 0;
            sW[L.tid] = L.tid >= from && L.tid < n ? sPw.f(L.tid < n ? n - 1 - L.tid : 0) * p.z_scale * (float)owed.inverse : 0.0f;
        }
        fetch(ch + 1);
        if (Cfg::NP == 1 && held) put_rows(ch - 1);
        barrier_lds();
        const bool bad = bad_z | pairs<Cfg>(sP, sX, sY, sAge, m, L);
        const uint64_t bads = __ballot(bad);
        if (L.lane == 0) sBad[L.w] = bads != 0;
        barrier_lds();
        L.again();
        uint32_t any_bad = 0;
#pragma unroll
        for (int i = 0; i < Cfg::W; ++i) any_bad |= sBad[i];
        held = Cfg::NP == 1 && os == 2 && any_bad == 0;

        if (__builtin_amdgcn_readfirstlane((int)any_bad) == 0) {
            // ---- the rows against the state before the chunk
            f32x4 acc[Cfg::NB];
#pragma unroll
            for (int ib = 0; ib < Cfg::NB; ++ib) acc[ib] = zero4();
#pragma unroll
            for (int s = 0; s < Cfg::KS; ++s) {
                bf16x8 st[Cfg::FP];
                planes8<Cfg::FP>(S[s][0], S[s][1], st);
#pragma unroll
                for (int ib = 0; ib < Cfg::NB; ++ib) {
                    bf16x8 x[Cfg::NP];
                    row_frag<Cfg, Cfg::KD>(x, sX, 16 * ib, s, L);
                    mma<Cfg::FP, Cfg::NP>(acc[ib], st, x);
                }
                // without a limit the scheduler reads all of x ahead, and the
                // registers of the next chunk's rows are spilled, which waits for them
                if (s % 2 == 1) __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int ib = 0; ib < Cfg::NB; ++ib) acc[ib] *= sPw.f(16 * ib + L.c + e) * before;
            if (m) {
#pragma unroll
                for (int ib = 0; ib < Cfg::NB; ++ib) {
                    const bool goes_on = (m & upto(16 * ib + L.c)) == 0;
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[ib][r] = goes_on ? acc[ib][r] : 0.0f;
                }
            }
            settle<Cfg>(S, m != 0, take, cy);
            fetch_z(ch + 1);                               // here, for the registers

            // ---- the rows against each other, and the state after the chunk
#pragma unroll
            for (int tb = 0; tb < Cfg::C / 32; ++tb) {
                bf16x8 z[Cfg::NP], zw[3];
                col_frag<Cfg, Cfg::VD>(z, sZ, tb, state_col_addr(L), L);
#pragma unroll
                for (int ib = 2 * tb; ib < Cfg::NB; ++ib) {
                    const int t0 = ib * (ib + 1) / 2 + 2 * tb;
                    bf16x8 pr[Cfg::FP];
#pragma unroll
                    for (int q = 0; q < Cfg::FP; ++q) {
                        const u32x2 lo = sP[t0][q][L.lane];
                        const u32x2 hi = ib > 2 * tb ? sP[t0 + (ib > 2 * tb ? 1 : 0)][q][L.lane] : u32x2{0u, 0u};
                        pr[q] = __builtin_bit_cast(bf16x8, u32x4{lo.x, lo.y, hi.x, hi.y});
                    }
                    mma<Cfg::NP, Cfg::FP>(acc[ib], z, pr);
                }
                weigh<Cfg>(zw, z, sW, tb, L);
#pragma unroll
                for (int s = 0; s < Cfg::KS; ++s)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        bf16x8 y[Cfg::NP];
                        col_frag<Cfg, Cfg::KD>(y, sY, tb, state_row_addr(s, u, L), L);
                        mma<Cfg::NP, 3>(S[s][u], y, zw);
                    }
            }

            // ---- out: four consecutive columns of a row per lane
            if (Cfg::NP == 1 && os == 2) {
#pragma unroll
                for (int ib = 0; ib < Cfg::NB; ++ib) {
                    const int row = 16 * ib + L.c, unit = 2 * L.w + (L.g >> 1);
                    *(u32x2*)(sO + row * Cfg::VD + swizzled<Cfg::VD>(unit, row) * 8 + 4 * (L.g & 1)) =
                        u32x2{f32x2_to_bf16x2(acc[ib][0], acc[ib][1]), f32x2_to_bf16x2(acc[ib][2], acc[ib][3])};
                }
            } else {
                const RetRows o = rows_out(ch);
#pragma unroll
                for (int ib = 0; ib < Cfg::NB; ++ib)
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[ib]), o.r,
                                                           (int)o.offset(16 * ib + L.c, 16 * L.w + 4 * L.g, 4), 0, 0);
            }
        } else {
            // ---- row by row
            const RetRows o = rows_out(ch);
            fetch_z(ch + 1);
            carry_state<Cfg>(S, Carry{was, 0.0f});
            owed.none();
            const Carry one = carry_by(sPw.of[1]);
#pragma unroll 1
            for (int i = 0; i < n; ++i) {
                const bool begin = (m >> i) & 1ull;
                const Carry by = i == 0 && e == 0 ? Carry{1.0f, 0.0f} : one;
                each<Cfg>(S, [&](float x, int, int, int) { return begin ? 0.0f : by(x); });
                const float z = tile_value<Cfg, Cfg::VD>(sZ, i, state_col(L)) * p.z_scale;
                float sum = 0.0f;
#pragma unroll
                for (int s = 0; s < Cfg::KS; ++s) {
                    float x[8], y[8];
                    row_values<Cfg, Cfg::KD>(x, sX, i, s, L);
                    row_values<Cfg, Cfg::KD>(y, sY, i, s, L);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        S[s][k >> 2][k & 3] = __builtin_fmaf(y[k], z, S[s][k >> 2][k & 3]);
                        sum = __builtin_fmaf(x[k], S[s][k >> 2][k & 3], sum);
                    }
                    __builtin_amdgcn_sched_barrier(0);     // few registers: the next chunk's rows hold theirs
                }
                sum += lanes_xor(sum, 16);
                sum += lanes_xor(sum, 32);
                sum *= p.inter_scale;
                const uint32_t off = L.g == 0 ? o.offset(i, state_col(L), os) : kOob;
                if (os == 2) __builtin_amdgcn_raw_buffer_store_b16((uint16_t)f32_to_bf16(sum), o.r, (int)off, 0, 0);
                else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(sum), o.r, (int)off, 0, 0);
            }
        }
    }
    if (Cfg::NP == 1 && held) {
        barrier_lds();
        put_rows(run.nch - 1);
    }
    if (p.fin && seg == (p.rev ? 0 : p.nseg - 1)) {
        // backwards: the gradient of the state before the tape, one step further
        // back, and none if step 0 begins an episode
        const bool drop = p.rev && start[0] != 0;
        store_state<Cfg>(S, p.fin + bh * words, p.sk, p.sv, p.x.d, p.z.d, (p.rev ? sPw.f(1) : 1.0f) * (float)owed.now, drop, L);
    }
}

// ------------------------------------------------------ gradients of shared heads
// Bound by memory: T = 32768, 32 query heads on 8 of 128, 240 us, 5.0 TB/s.
template <int NP>
__global__ __launch_bounds__(256) void ret_share_kernel(RetShareArgs p) {
    const RetShareArgs::Part& a = blockIdx.y ? p.v : p.k;
    const int64_t units = p.rows * (a.d / 4);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < units; i += (int64_t)gridDim.x * 256) {
        const int64_t rk = i / (a.d / 4), c = i % (a.d / 4);   // (step, key head), four columns
        const f32x4* const x = (const f32x4*)a.part + rk * p.G * (a.d / 4) + c;
        f32x4 s = x[0];
        for (int g = 1; g < p.G; ++g) s += x[(int64_t)g * (a.d / 4)];
        if (NP == 1) ((u32x2*)a.out)[i] = u32x2{f32x2_to_bf16x2(s[0], s[1]), f32x2_to_bf16x2(s[2], s[3])};
        else ((f32x4*)a.out)[i] = s;
    }
}

// ------------------------------------------------------------------- launches
namespace {
// f(Cfg) for the smallest tile that holds the state's kd rows and vd columns
template <int NP, class F>
void with_tiles(int kd, int vd, F&& f) {
    if (kd <= 64) {
        if (vd <= 64) f(RetCfg<NP, 64, 64>{});
        else f(RetCfg<NP, 64, 128>{});
    } else {
        if (vd <= 64) f(RetCfg<NP, 128, 64>{});
        else f(RetCfg<NP, 128, 128>{});
    }
}
template <class F>
void with_cfg(int planes, int kd, int vd, F&& f) {
    if (planes == 1) with_tiles<1>(kd, vd, f);
    else with_tiles<3>(kd, vd, f);
}
}  // namespace

hipError_t ret_walk_launch(int planes, RetWalkSet set, int64_t B, hipStream_t s) {
    const RetWalkArgs& a = set.w[0];
    set.B = B;
    set.tasks = B * a.H * a.nseg;
    set.blocks = (set.tasks + 7) / 8 * 8 * set.n;
    const dim3 grid((unsigned)(set.blocks + (set.grad_alpha ? a.H : 0)));
    with_cfg(planes, a.x.d, a.z.d, [&](auto cfg) {
        using Cfg = decltype(cfg);
        hipLaunchKernelGGL((ret_walk_kernel<Cfg>), grid, dim3(Cfg::THREADS), 0, s, set);
    });
    return hipGetLastError();
}
bool ret_same_tiles(int64_t kd0, int64_t vd0, int64_t kd1, int64_t vd1) {
    return (kd0 <= 64) == (kd1 <= 64) && (vd0 <= 64) == (vd1 <= 64);
}

hipError_t ret_summary_launch(int planes, const RetSummaryArgs& a, int64_t B, hipStream_t s) {
    const dim3 grid((unsigned)(a.nseg - 1), (unsigned)a.H, (unsigned)B);
    with_cfg(planes, a.y.d, a.z.d, [&](auto cfg) {
        using Cfg = decltype(cfg);
        hipLaunchKernelGGL((ret_summary_kernel<Cfg>), grid, dim3(Cfg::THREADS), 0, s, a);
    });
    return hipGetLastError();
}

hipError_t ret_prep_launch(int planes, const RetPrepArgs& a, int64_t B, hipStream_t s) {
    const dim3 grid((unsigned)a.nseg, (unsigned)a.H, (unsigned)B);
    with_cfg(planes, a.q.d, a.v.d, [&](auto cfg) {
        using Cfg = RetCfg64<decltype(cfg)>;
        if (a.dstates) hipLaunchKernelGGL((ret_prep_kernel<Cfg, true>), grid, dim3(Cfg::THREADS), 0, s, a);
        else hipLaunchKernelGGL((ret_prep_kernel<Cfg, false>), grid, dim3(Cfg::THREADS), 0, s, a);
    });
    return hipGetLastError();
}

namespace {
// One group where there are few segments or many columns, else 32
bool scan_one_group(int64_t words, int64_t heads, int64_t n) { return n <= 16 || heads * (words / 4) >= 16384; }
template <int GROUPS, int RPT, bool DOT>
void state_scan(const RetStateScanArgs& a, const RetStateScanArgs* back, int64_t B, hipStream_t s) {
    constexpr int kCols = 256 / GROUPS;
    const dim3 grid((unsigned)((a.words / 4 + kCols - 1) / kCols), (unsigned)a.H, (unsigned)(back ? 2 * B : B));
    hipLaunchKernelGGL((ret_state_scan_kernel<GROUPS, RPT, DOT>), grid, dim3(256), 0, s, a, back ? *back : a, (int)B);
}
template <bool DOT>
void state_scan_for(const RetStateScanArgs& a, const RetStateScanArgs* back, int64_t B, hipStream_t s) {
    const int n = DOT ? a.nseg : a.nseg - 1;
    if (!scan_one_group(a.words, B * a.H, a.nseg)) {
        if (n <= 64) state_scan<32, 2, DOT>(a, back, B, s);
        else state_scan<32, 4, DOT>(a, back, B, s);
    } else if (n <= 4) {
        state_scan<1, 4, DOT>(a, back, B, s);
    } else {
        state_scan<1, 16, DOT>(a, back, B, s);
    }
}
}  // namespace

int64_t ret_scan_parts(int64_t words, int64_t heads, int64_t nseg) {
    const int64_t cols = scan_one_group(words, heads, nseg) ? 256 : 256 / 32;
    return (words / 4 + cols - 1) / cols;
}

hipError_t ret_state_scan_launch(const RetStateScanArgs& a, const RetStateScanArgs* back, int64_t B, hipStream_t s) {
    if (a.dstates) state_scan_for<true>(a, back, B, s);
    else state_scan_for<false>(a, back, B, s);
    return hipGetLastError();
}

hipError_t ret_share_launch(int planes, const RetShareArgs& a, hipStream_t s) {
    const int64_t units = a.rows * ((a.k.d > a.v.d ? a.k.d : a.v.d) / 4), blocks = (units + 255) / 256;
    const dim3 grid((unsigned)(blocks < 8192 ? blocks : 8192), 2), block(256);
    if (planes == 1) hipLaunchKernelGGL((ret_share_kernel<1>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((ret_share_kernel<3>), grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace memoroid
