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
// decay in float and goes into the state as three planes, exactly (two, right to
// 2^-18, where no state of bf16 inputs comes out).  With bf16
// inputs P and the S that a row is multiplied with are rounded to bf16 once
// each, as operands: together they add to the output's own rounding what one
// more rounding would (1.4 times its error), and the state itself takes neither.
//
// A value that is not finite must not reach other episodes, nor earlier rows of
// its own, through a zero of P or of the decays (0 * NaN): a chunk that holds one
// is walked row by row, by the recurrence itself in floats.
#include "retention_common.hpp"

#include <type_traits>

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
__device__ __forceinline__ RetRows rows_of(const Head& x, int64_t w0, int n, int64_t T, bool rev) {
    return ret_rows(x.p, x.row_bytes, x.d, Cfg::ES, w0, n, T, rev);
}

// the value operand times a weight per row, in planes
template <class Cfg, int ZP>
__device__ __forceinline__ void weigh(bf16x8 (&out)[ZP], const bf16x8 (&z)[Cfg::NP], const float* w, int tb,
                                      const RetLane& L) {
    f32x4 lo = *(const f32x4*)(w + 32 * tb + 4 * L.g), hi = *(const f32x4*)(w + 32 * tb + 16 + 4 * L.g);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        lo[e] *= plane_value<Cfg::NP>(z, e);
        hi[e] *= plane_value<Cfg::NP>(z, e + 4);
    }
    planes8<ZP>(lo, hi, out);
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
// begin on.  DOT: also its derivative by log gamma, sum (n-1-j) gamma^(n-1-j) y^T z.
template <class Cfg, int ZP, bool DOT>
__global__ __launch_bounds__(Cfg::THREADS, 4) void ret_summary_kernel(RetSummaryArgs p) {
    __shared__ __attribute__((aligned(16))) uint16_t sY[Cfg::NP * Cfg::C * Cfg::KD];
    __shared__ __attribute__((aligned(16))) uint16_t sZ[Cfg::NP * Cfg::C * Cfg::VD];
    __shared__ Powers<Cfg::C + 1> sPw;
    __shared__ __attribute__((aligned(16))) float sW[DOT ? 2 : 1][Cfg::C];
    RetLane L;
    const int64_t seg = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    ret_header(p.hdr, p.sig);
    const double rate = fabs((double)p.alpha[h]);
    sPw.fill(rate, L.tid);
    const Head hy = head_of<Cfg>(p.y, b, h, p.T), hz = head_of<Cfg>(p.z, b, h, p.T);
    const uint8_t* const start = p.start + b * p.T;
    State<Cfg> S, D;
    zero_state<Cfg>(S);
    if (DOT) zero_state<Cfg>(D);
    Owed owed;
    __syncthreads();                                       // the powers are there
    bool any = false;
    RetTile<Cfg, Cfg::KD> ty;
    RetTile<Cfg, Cfg::VD> tz;
    uint32_t flag;
    // every segment here is a whole one: C rows per chunk (the last fetch, of a
    // chunk that is not there, reads nothing)
    auto fetch = [&](int ch) {
        const bool have = ch < p.chunks;
        const int w0 = have ? ((int)seg * p.chunks + ch) * Cfg::C : 0, n = have ? Cfg::C : 0;
        flag = ret_flag(start, w0, n, p.T, p.rev, L.lane);
        ty.fetch(rows_of<Cfg>(hy, w0, n, p.T, p.rev), L);
        tz.fetch(rows_of<Cfg>(hz, w0, n, p.T, p.rev), L);
    };
    fetch(0);
#pragma unroll 1
    for (int ch = 0; ch < p.chunks; ++ch) {
        L.again();
        const uint64_t m = __ballot(flag != 0u);
        const int from = m ? last_begin(m) : 0;
        any = any || m != 0;
        bool take = false;
        if (m) owed.none();
        else take = owed.add(sPw, Cfg::C);
        const Carry cy = carry_by(owed.now);
        if (take) owed.none();
        barrier_lds();                                     // the last chunk's operands have been read
        ty.stage(sY, from, L);
        tz.stage(sZ, from, L);
        if (L.tid < Cfg::C) {
            const int age = Cfg::C - 1 - L.tid;
            const float w = L.tid >= from ? sPw.f(age) * p.z_scale * (float)owed.inverse : 0.0f;
            sW[0][L.tid] = w;
            if (DOT) sW[DOT ? 1 : 0][L.tid] = w * (float)age;
        }
        fetch(ch + 1);
        barrier_lds();
        // d(gamma^C S)/dlog gamma = gamma^C (D + C S)
        if (DOT) {
            each<Cfg>(D, [&](float x, int s, int u, int e) { return __builtin_fmaf((float)Cfg::C, S[s][u][e], x); });
            settle<Cfg>(D, m != 0, take, cy);
        }
        settle<Cfg>(S, m != 0, take, cy);
#pragma unroll
        for (int tb = 0; tb < Cfg::C / 32; ++tb) {
            bf16x8 z[Cfg::NP], zw[ZP], zd[ZP];
            col_frag<Cfg, Cfg::VD>(z, sZ, tb, state_col_addr(L), L);
            weigh<Cfg, ZP>(zw, z, sW[0], tb, L);
            if (DOT) weigh<Cfg, ZP>(zd, z, sW[DOT ? 1 : 0], tb, L);
#pragma unroll
            for (int s = 0; s < Cfg::KS; ++s)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    bf16x8 y[Cfg::NP];
                    col_frag<Cfg, Cfg::KD>(y, sY, tb, state_row_addr(s, u, L), L);
                    mma<Cfg::NP, ZP>(S[s][u], y, zw);
                    if (DOT) mma<Cfg::NP, ZP>(D[s][u], y, zd);
                }
        }
    }
    L.again();
    const int64_t words = (int64_t)p.y.d * p.z.d, n = p.nseg - 1;
    const int64_t at = ((b * p.H + h) * n + seg) * words;
    store_state<Cfg>(S, p.states + at, p.z.d, 1, p.y.d, p.z.d, (float)owed.now, false, L);
    if (DOT) store_state<Cfg>(D, p.dstates + at, p.z.d, 1, p.y.d, p.z.d, (float)owed.now, false, L);
    if (h == 0 && L.tid == 0) p.R[b * n + seg] = any ? 1 : 0;
}

// ---------------------------------------------------------------- state scan
// states[i] becomes the state after segment i: its summary, plus gamma^rows times
// the state before it where it holds no begin step; with DOT the derivative
// likewise, d' = own + gamma^rows (d + rows s).  GROUPS threads share a 16-byte
// column of the states, each with RPT consecutive segments of it in registers, all
// loads in flight at once; the groups combine through LDS.  One read and one write
// of the states.  One group where there are few segments or many columns (3
// segments of 128 heads of 128 x 128: 10 us, 294 us in 32 groups; 31 segments of 16
// such heads: 16 and 53 us), else 32 (128 segments of 4 heads of 64 x 64: 8 us, 39 us
// one segment after the other).
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
__global__ __launch_bounds__(256) void ret_state_scan_kernel(RetStateScanArgs p) {
    constexpr int kCols = 256 / GROUPS, kTile = GROUPS * RPT;
    __shared__ f32x4 sTot[GROUPS > 1 && DOT ? 2 : 1][GROUPS][GROUPS > 1 ? kCols : 1];
    __shared__ uint32_t sFlag[GROUPS];
    const int col = threadIdx.x % kCols, grp = threadIdx.x / kCols;
    const int64_t h = blockIdx.y, b = blockIdx.z, bh = b * p.H + h;
    const int c4 = (int)blockIdx.x * kCols + col, w4 = p.words / 4;   // words is a multiple of 64
    const bool in = c4 < w4;
    const double rate = fabs((double)p.alpha[h]), rows = (double)p.rows;
    const Carry one = carry_of(rate, rows), many = carry_of(rate, rows * RPT);
    // backwards the seed belongs to the last step itself: one decay less
    const Carry one0 = p.rev ? carry_of(rate, rows - 1.0) : one, many0 = p.rev ? carry_of(rate, rows * RPT - 1.0) : many;
    f32x4* const S = (f32x4*)p.states + bh * p.n * w4 + c4;
    f32x4* const D = DOT ? (f32x4*)p.dstates + bh * p.n * w4 + c4 : nullptr;
    const uint8_t* const R = p.R + b * p.n;
    const f32x4 zero = zero4();
    SegState<DOT> before;                                  // the state before the tile
    if (p.seed && in) before.s = ((const f32x4*)p.seed)[bh * w4 + c4];
    for (int base = 0; base < p.n; base += kTile) {
        f32x4 x[RPT], y[DOT ? RPT : 1];
        bool fl[RPT];
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int l = base + grp * RPT + i;
            const bool have = in && l < p.n;
            x[i] = have ? S[(int64_t)l * w4] : zero;
            if (DOT) y[DOT ? i : 0] = have ? D[(int64_t)l * w4] : zero;
            fl[i] = l < p.n && R[l < p.n ? l : 0] != 0;
        }
        SegState<DOT> mine = before;                       // the state before this thread's run
        if constexpr (GROUPS > 1) {
            SegState<DOT> tot;
            bool any = false;
#pragma unroll
            for (int i = 0; i < RPT; ++i) {
                tot.then(x[i], y[DOT ? i : 0], fl[i], one, (float)p.rows);
                any |= fl[i];
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
            mine.then(x[i], y[DOT ? i : 0], fl[i], l == 0 ? one0 : one, (float)p.rows);
            if (in && l < p.n) {
                S[(int64_t)l * w4] = mine.s;
                if (DOT) D[(int64_t)l * w4] = mine.d;
            }
        }
        if constexpr (GROUPS == 1) before = mine;
    }
}

// ---------------------------------------------------------------------- walk
// The masked, decayed products of a chunk's rows in tiles as operands of the next
// product, a tile or two per wavefront.  by_age[16 + n]: the weight of a partner n
// steps back, 0 for n < 0;  m: begin bits.  Returns whether a row's
// product with itself came out not finite: every x and y that is not finite shows
// there (and so does one that overflows).
template <class Cfg>
__device__ __forceinline__ bool pairs(u32x2 (&sP)[Cfg::NTILE][Cfg::NP][64], const uint16_t* sX, const uint16_t* sY,
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
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (ib == jb) bad |= age == r && !(fabsf(d[r]) < __builtin_inff());
            d[r] *= by_age[age - r + 16];
        }
        if (m) {                                                           // age of the row's first partner
            const uint64_t mr = m & upto(row);
            const int oldest = mr ? row - last_begin(mr) : row;
#pragma unroll
            for (int r = 0; r < 4; ++r) d[r] = age - r <= oldest ? d[r] : 0.0f;
        }
        uint32_t lo[Cfg::NP], hi[Cfg::NP];
        planes2<Cfg::NP>(d[0], d[1], lo);
        planes2<Cfg::NP>(d[2], d[3], hi);
#pragma unroll
        for (int q = 0; q < Cfg::NP; ++q) sP[idx][q][L.lane] = u32x2{lo[q], hi[q]};
    }
    return bad;
}

template <class Cfg, int ZP>
__global__ __launch_bounds__(Cfg::THREADS, Cfg::KD == 64 || Cfg::VD == 128 ? 4 : 3) void ret_walk_kernel(RetWalkArgs p) {
    __shared__ __attribute__((aligned(16))) uint16_t sX[Cfg::NP * Cfg::C * Cfg::KD];
    __shared__ __attribute__((aligned(16))) uint16_t sY[Cfg::NP * Cfg::C * Cfg::KD];
    __shared__ __attribute__((aligned(16))) uint16_t sZ[Cfg::NP * Cfg::C * Cfg::VD];
    // bf16 out: rows gathered here, so that they leave 16 bytes a lane, a row at a
    // time (a wavefront's own 32 bytes of a row doubled the bytes written)
    __shared__ __attribute__((aligned(16))) uint16_t sO[Cfg::NP == 1 ? Cfg::C * Cfg::VD : 8];
    __shared__ u32x2 sP[Cfg::NTILE][Cfg::NP][64];
    __shared__ Powers<Cfg::C + 1> sPw;
    __shared__ float sAge[Cfg::C + 16];
    __shared__ __attribute__((aligned(16))) float sW[Cfg::C];
    __shared__ uint32_t sBad[Cfg::W];
    RetLane L;
    const int64_t seg = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    ret_header(p.hdr, p.sig);
    const double rate = fabs((double)p.alpha[h]);
    sPw.fill(rate, L.tid);
    if (L.tid < Cfg::C + 16) sAge[L.tid] = L.tid < 16 ? 0.0f : decay_pow(rate, L.tid - 16) * p.p_scale;
    const Head hx = head_of<Cfg>(p.x, b, h, p.T), hy = head_of<Cfg>(p.y, b, h, p.T), hz = head_of<Cfg>(p.z, b, h, p.T);
    const uint8_t* const start = p.start + b * p.T;
    const int64_t words = (int64_t)p.x.d * p.z.d, bh = b * p.H + h;
    const int T = (int)p.T, seg0 = (int)seg * p.chunks * Cfg::C;
    const int left = (T - seg0 + Cfg::C - 1) / Cfg::C, nch = left < p.chunks ? left : p.chunks;
    const int os = Cfg::NP == 1 && !p.out_f32 ? 2 : 4;
    auto rows_in = [&](int ch) {                           // rows of chunk ch, none past the segment
        const int rest = ch < nch ? T - (seg0 + ch * Cfg::C) : 0;
        return rest < Cfg::C ? rest : Cfg::C;
    };
    auto first_of = [&](int ch) { return ch < nch ? seg0 + ch * Cfg::C : 0; };
    auto rows_out = [&](int ch) {
        return ret_rows((char*)p.out + (b * p.T * p.H + h) * p.z.d * os, (int64_t)p.H * p.z.d * os, p.z.d, os, first_of(ch),
                        rows_in(ch), p.T, p.rev);
    };

    RetTile<Cfg, Cfg::KD> tx, ty;
    RetTile<Cfg, Cfg::VD> tz;
    uint32_t flag;
    auto fetch = [&](int ch) {
        const int w0 = first_of(ch), n = rows_in(ch);
        flag = ret_flag(start, w0, n, p.T, p.rev, L.lane);
        tx.fetch(rows_of<Cfg>(hx, w0, n, p.T, p.rev), L);
        ty.fetch(rows_of<Cfg>(hy, w0, n, p.T, p.rev), L);
    };
    auto fetch_z = [&](int ch) { tz.fetch(rows_of<Cfg>(hz, first_of(ch), rows_in(ch), p.T, p.rev), L); };
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
    load_state<Cfg>(S, seg == 0 ? (p.seed ? p.seed + bh * words : nullptr) : p.states + (bh * (p.nseg - 1) + seg - 1) * words,
                    p.sk, p.sv, p.x.d, p.z.d, L);
#pragma unroll 1
    for (int ch = 0; ch < nch; ++ch) {
        L.again();
        const int n = rows_in(ch);
        const uint64_t m = __ballot(flag != 0u);
        const bool bad_z = tz.bad() != 0u;
        // the gradient of the state after the tape belongs to the last step
        const int e = p.rev && seg == 0 && ch == 0 ? 0 : 1;
        const float was = uniform((float)owed.now), before = was * p.inter_scale;
        bool take = false;
        if (m) owed.none();
        else take = owed.add(sPw, n - 1 + e);
        const Carry cy = carry_by(owed.now);
        if (take) owed.none();
        barrier_lds();                                     // the last chunk's operands have been read
        tx.stage(sX, 0, L);
        ty.stage(sY, 0, L);
        tz.stage(sZ, 0, L);
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
                bf16x8 st[Cfg::NP];
                planes8<Cfg::NP>(S[s][0], S[s][1], st);
#pragma unroll
                for (int ib = 0; ib < Cfg::NB; ++ib) {
                    bf16x8 x[Cfg::NP];
                    row_frag<Cfg, Cfg::KD>(x, sX, 16 * ib, s, L);
                    mma<Cfg::NP, Cfg::NP>(acc[ib], st, x);
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
                bf16x8 z[Cfg::NP], zw[ZP];
                col_frag<Cfg, Cfg::VD>(z, sZ, tb, state_col_addr(L), L);
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
                    mma<Cfg::NP, Cfg::NP>(acc[ib], z, pr);
                }
                weigh<Cfg, ZP>(zw, z, sW, tb, L);
#pragma unroll
                for (int s = 0; s < Cfg::KS; ++s)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        bf16x8 y[Cfg::NP];
                        col_frag<Cfg, Cfg::KD>(y, sY, tb, state_row_addr(s, u, L), L);
                        mma<Cfg::NP, ZP>(S[s][u], y, zw);
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
        put_rows(nch - 1);
    }
    if (p.fin && seg == p.nseg - 1) {
        // backwards: the gradient of the state before the tape, one step further
        // back, and none if step 0 begins an episode
        const bool drop = p.rev && start[0] != 0;
        store_state<Cfg>(S, p.fin + bh * words, p.sk, p.sv, p.x.d, p.z.d, (p.rev ? sPw.f(1) : 1.0f) * (float)owed.now, drop, L);
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
__global__ __launch_bounds__(Cfg::THREADS, 2) void ret_sens_kernel(RetSensArgs p) {
    __shared__ __attribute__((aligned(16))) uint16_t sQ[Cfg::NP * Cfg::C * Cfg::KD];
    __shared__ __attribute__((aligned(16))) uint16_t sK[Cfg::NP * Cfg::C * Cfg::KD];
    __shared__ __attribute__((aligned(16))) uint16_t sV[Cfg::NP * Cfg::C * Cfg::VD];
    __shared__ __attribute__((aligned(16))) uint16_t sG[Cfg::NP * Cfg::C * Cfg::VD];
    __shared__ Powers<Cfg::C + 1> sPw;
    __shared__ float sAge[Cfg::C + 16];                    // [16 + n]: n gamma^n scale, 0 for n < 0
    __shared__ __attribute__((aligned(16))) float sW[4][Cfg::C];
    __shared__ uint32_t sBad[Cfg::W];
    __shared__ double sSum[Cfg::W];
    RetLane L;
    const int64_t seg = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    const double rate = fabs((double)p.alpha[h]);
    sPw.fill(rate, L.tid);
    if (L.tid < Cfg::C + 16) {
        const int age = L.tid - 16;
        sAge[L.tid] = age < 0 ? 0.0f : decay_pow(rate, age) * (float)age * p.scale;
    }
    const int kd = p.q.d, vd = p.v.d;
    const Head hq = head_of<Cfg>(p.q, b, h, p.T), hk = head_of<Cfg>(p.k, b, h, p.T), hv = head_of<Cfg>(p.v, b, h, p.T),
               hg = head_of<Cfg>(p.g, b, h, p.T);
    const uint8_t* const start = p.start + b * p.T;
    const int64_t words = (int64_t)kd * vd, bh = b * p.H + h;
    const int T = (int)p.T, seg0 = (int)seg * p.chunks * Cfg::C;
    const int left = (T - seg0 + Cfg::C - 1) / Cfg::C, nch = left < p.chunks ? left : p.chunks;

    RetTile<Cfg, Cfg::KD> tq, tk;
    RetTile<Cfg, Cfg::VD> tv, tg;
    uint32_t flag;
    auto fetch = [&](int ch) {
        const bool have = ch < nch;
        const int w0 = have ? seg0 + ch * Cfg::C : 0, rest = have ? T - w0 : 0, n = rest < Cfg::C ? rest : Cfg::C;
        flag = ret_flag(start, w0, n, p.T, false, L.lane);
        tq.fetch(rows_of<Cfg>(hq, w0, n, p.T, false), L);
        tk.fetch(rows_of<Cfg>(hk, w0, n, p.T, false), L);
        tv.fetch(rows_of<Cfg>(hv, w0, n, p.T, false), L);
        tg.fetch(rows_of<Cfg>(hg, w0, n, p.T, false), L);
    };
    fetch(0);
    State<Cfg> S, D;
    const int64_t at = (bh * (p.nseg - 1) + seg - 1) * words;
    load_state<Cfg>(S, seg == 0 ? (p.seed ? p.seed + bh * words : nullptr) : p.states + at, vd, 1, kd, vd, L);
    load_state<Cfg>(D, seg == 0 ? nullptr : p.dstates + at, vd, 1, kd, vd, L);
    Owed owed;
    __syncthreads();                                       // the powers are there
    double sum = 0.0;
#pragma unroll 1
    for (int ch = 0; ch < nch; ++ch) {
        L.again();
        const int rest = T - (seg0 + ch * Cfg::C), n = rest < Cfg::C ? rest : Cfg::C;
        const uint64_t m = __ballot(flag != 0u);
        const float before = uniform((float)owed.now);
        bool take = false;
        if (m) owed.none();
        else take = owed.add(sPw, n);
        const Carry cy = carry_by(owed.now);
        if (take) owed.none();
        const uint64_t not_finite = __ballot((tq.bad() | tk.bad() | tv.bad() | tg.bad()) != 0u);
        barrier_lds();                                     // the last operands have been read
        if (L.lane == 0) sBad[L.w] = not_finite != 0;
        tq.stage(sQ, 0, L);
        tk.stage(sK, 0, L);
        tv.stage(sV, 0, L);
        tg.stage(sG, 0, L);
        if (L.tid < Cfg::C) {
            const int i = L.tid;
            const int from = m ? last_begin(m) : 0;
            const float w = i < n && i >= from ? sPw.f(i < n ? n - 1 - i : 0) * (float)owed.inverse : 0.0f;
            sW[0][i] = w;
            sW[1][i] = w * (float)(n - 1 - i);
            const float f = i < n && (m & upto(i)) == 0 ? sPw.f(i + 1) * p.scale * before : 0.0f;
            sW[2][i] = f;
            sW[3][i] = f * (float)(i + 1);
        }
        fetch(ch + 1);
        barrier_lds();
        uint32_t any_bad = 0;
#pragma unroll
        for (int i = 0; i < Cfg::W; ++i) any_bad |= sBad[i];
        float part = 0.0f;
        if (__builtin_amdgcn_readfirstlane((int)any_bad) == 0) {
#pragma unroll
            for (int i = 0; i < (Cfg::NTILE + Cfg::W - 1) / Cfg::W; ++i) {
                const int idx = Cfg::W * i + L.w;
                if (idx >= Cfg::NTILE) break;
                int jb, ib;
                tile_of(idx, jb, ib);
                const f32x4 x = pair_products<Cfg, Cfg::KD>(sK, sQ, jb, ib, L);
                const f32x4 y = pair_products<Cfg, Cfg::VD>(sV, sG, jb, ib, L);
                const int row = 16 * ib + L.c, age = row - 16 * jb - 4 * L.g;
                const uint64_t mr = m & upto(row);
                const int oldest = mr ? row - last_begin(mr) : row;
#pragma unroll
                for (int r = 0; r < 4; ++r) part += age - r <= oldest ? x[r] * y[r] * sAge[age - r + 16] : 0.0f;
            }
            // rows against (S, D): skipped where the first row begins an episode,
            // so that values of S that are not finite stay out
            if (!(m & 1ull)) {
                bf16x8 g1[Cfg::C / 32][3], g2[Cfg::C / 32][3];
#pragma unroll
                for (int tb = 0; tb < Cfg::C / 32; ++tb) {
                    bf16x8 g[Cfg::NP];
                    col_frag<Cfg, Cfg::VD>(g, sG, tb, state_col_addr(L), L);
                    weigh<Cfg, 3>(g1[tb], g, sW[2], tb, L);
                    weigh<Cfg, 3>(g2[tb], g, sW[3], tb, L);
                }
#pragma unroll
                for (int s = 0; s < Cfg::KS; ++s)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        f32x4 o1 = zero4(), o2 = zero4();
#pragma unroll
                        for (int tb = 0; tb < Cfg::C / 32; ++tb) {
                            bf16x8 q[Cfg::NP];
                            col_frag<Cfg, Cfg::KD>(q, sQ, tb, state_row_addr(s, u, L), L);
                            mma<Cfg::NP, 3>(o1, q, g1[tb]);
                            mma<Cfg::NP, 3>(o2, q, g2[tb]);
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            part = __builtin_fmaf(S[s][u][e], o2[e], __builtin_fmaf(D[s][u][e], o1[e], part));
                    }
            }
            // (S, D) after the chunk
            each<Cfg>(D, [&](float x, int s, int u, int e) { return __builtin_fmaf((float)n, S[s][u][e], x); });
            settle<Cfg>(D, m != 0, take, cy);
            settle<Cfg>(S, m != 0, take, cy);
#pragma unroll
            for (int tb = 0; tb < Cfg::C / 32; ++tb) {
                bf16x8 z[Cfg::NP], zw[3], zd[3];
                col_frag<Cfg, Cfg::VD>(z, sV, tb, state_col_addr(L), L);
                weigh<Cfg, 3>(zw, z, sW[0], tb, L);
                weigh<Cfg, 3>(zd, z, sW[1], tb, L);
#pragma unroll
                for (int s = 0; s < Cfg::KS; ++s)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        bf16x8 y[Cfg::NP];
                        col_frag<Cfg, Cfg::KD>(y, sK, tb, state_row_addr(s, u, L), L);
                        mma<Cfg::NP, 3>(S[s][u], y, zw);
                        mma<Cfg::NP, 3>(D[s][u], y, zd);
                    }
            }
        } else {
            // ---- row by row
            carry_state<Cfg>(S, Carry{before, 0.0f});
            carry_state<Cfg>(D, Carry{before, 0.0f});
            owed.none();
            const Carry one = carry_by(sPw.of[1]);
#pragma unroll 1
            for (int i = 0; i < n; ++i) {
                const bool begin = (m >> i) & 1ull;
                each<Cfg>(D, [&](float x, int s, int u, int e) { return begin ? 0.0f : one(x + S[s][u][e]); });
                each<Cfg>(S, [&](float x, int, int, int) { return begin ? 0.0f : one(x); });
                const float v = tile_value<Cfg, Cfg::VD>(sV, i, state_col(L));
                float dot = 0.0f;
#pragma unroll
                for (int s = 0; s < Cfg::KS; ++s) {
                    float q[8], k[8];
                    row_values<Cfg, Cfg::KD>(q, sQ, i, s, L);
                    row_values<Cfg, Cfg::KD>(k, sK, i, s, L);
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                        S[s][x >> 2][x & 3] = __builtin_fmaf(k[x], v, S[s][x >> 2][x & 3]);
                        dot = __builtin_fmaf(q[x], D[s][x >> 2][x & 3], dot);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                // (nothing where the row begins: 0 times what is not finite stays out)
                if (!begin) part = __builtin_fmaf(dot * p.scale, tile_value<Cfg, Cfg::VD>(sG, i, state_col(L)), part);
            }
        }
        sum += (double)part;
    }
    L.again();
    if (p.grad_state && seg == p.nseg - 1) {
        State<Cfg> G;
        load_state<Cfg>(G, p.grad_state + bh * words, vd, 1, kd, vd, L);
        each<Cfg>(G, [&](float x, int s, int u, int e) {
            sum += (double)D[s][u][e] * (double)x * owed.now;
            return x;
        });
    }
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x, 64);
    if (L.lane == 0) sSum[L.w] = sum;
    __syncthreads();
    if (L.tid == 0) {
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < Cfg::W; ++i) s += sSum[i];
        p.part[bh * p.nseg + seg] = s;
    }
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
// the planes of z: three, or two where bf16's state stays inside (kernels.hpp)
template <class Cfg, class F>
void with_planes(bool exact, F&& f) {
    if constexpr (Cfg::NP == 1) {
        if (!exact) {
            f(std::integral_constant<int, 2>{});
            return;
        }
    }
    f(std::integral_constant<int, 3>{});
}
}  // namespace

hipError_t ret_walk_launch(int planes, const RetWalkArgs& a, int64_t B, hipStream_t s) {
    const dim3 grid((unsigned)a.nseg, (unsigned)a.H, (unsigned)B);
    with_cfg(planes, a.x.d, a.z.d, [&](auto cfg) {
        using Cfg = decltype(cfg);
        with_planes<Cfg>(a.exact, [&](auto zp) {
            hipLaunchKernelGGL((ret_walk_kernel<Cfg, decltype(zp)::value>), grid, dim3(Cfg::THREADS), 0, s, a);
        });
    });
    return hipGetLastError();
}

hipError_t ret_summary_launch(int planes, const RetSummaryArgs& a, int64_t B, hipStream_t s) {
    const dim3 grid((unsigned)(a.nseg - 1), (unsigned)a.H, (unsigned)B);
    with_cfg(planes, a.y.d, a.z.d, [&](auto cfg) {
        using Cfg = decltype(cfg);
        const dim3 block(Cfg::THREADS);
        if (a.dstates)
            hipLaunchKernelGGL((ret_summary_kernel<Cfg, 3, true>), grid, block, 0, s, a);
        else
            with_planes<Cfg>(a.exact, [&](auto zp) {
                hipLaunchKernelGGL((ret_summary_kernel<Cfg, decltype(zp)::value, false>), grid, block, 0, s, a);
            });
    });
    return hipGetLastError();
}

namespace {
template <int GROUPS, int RPT, bool DOT>
void state_scan(const RetStateScanArgs& a, int64_t B, hipStream_t s) {
    constexpr int kCols = 256 / GROUPS;
    const dim3 grid((unsigned)((a.words / 4 + kCols - 1) / kCols), (unsigned)a.H, (unsigned)B);
    hipLaunchKernelGGL((ret_state_scan_kernel<GROUPS, RPT, DOT>), grid, dim3(256), 0, s, a);
}
template <bool DOT>
void state_scan_for(const RetStateScanArgs& a, int64_t B, hipStream_t s) {
    const int64_t columns = B * a.H * (a.words / 4);
    if (a.n <= 4) state_scan<1, 4, DOT>(a, B, s);
    else if (a.n <= 16 || columns >= 16384) state_scan<1, 16, DOT>(a, B, s);
    else if (a.n <= 64) state_scan<32, 2, DOT>(a, B, s);
    else state_scan<32, 4, DOT>(a, B, s);
}
}  // namespace

hipError_t ret_state_scan_launch(const RetStateScanArgs& a, int64_t B, hipStream_t s) {
    if (a.dstates) state_scan_for<true>(a, B, s);
    else state_scan_for<false>(a, B, s);
    return hipGetLastError();
}

hipError_t ret_sens_launch(int planes, const RetSensArgs& a, int64_t B, hipStream_t s) {
    const dim3 grid((unsigned)a.nseg, (unsigned)a.H, (unsigned)B);
    with_cfg(planes, a.q.d, a.v.d, [&](auto cfg) {
        using Cfg = decltype(cfg);
        hipLaunchKernelGGL((ret_sens_kernel<Cfg>), grid, dim3(Cfg::THREADS), 0, s, a);
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
