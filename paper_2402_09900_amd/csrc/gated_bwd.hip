// gated_bwd.hip -- gradient of the gated recurrence, in one pass over memory.
//
// With g = dL/dh and lam = dL/dh with what later steps add,
//     lam_t = g_t + c_t,   c_{t-1} = a_t lam_t  (0 at a begin step; the last c: dL/dstate),
//     dx = lam m sig(i),   di = lam b (1 - sig(i)),
//     du = lam a (sig(i) x a / m - h_before),   dr = du u (1 - sig(r)),
//     dalpha = sign(alpha) sum du sig(r).
// A tile is 128 steps: the forward call has kept the state before each, so h is run through
// again within a tile and only c goes from tile to tile, the last first.  Otherwise
// as forward (gated_fwd.hip): the runs' effects on h and on c, put one behind the other
// by a wavefront each; then h through each run; then, with the c that enters, back through
// it, forming every gradient.  Sums for dalpha: a row per tile, added up by a second
// kernel in doubles.
#include <type_traits>

#include "gated_common.hpp"

namespace memoroid {

namespace {

template <bool BF16, bool FULL, int F, int L, int THREADS, int WAVES>
__global__ __launch_bounds__(THREADS, WAVES) void gated_bwd_kernel(GatedBwdArgs p) {
    constexpr int kRow = Lanes<F, THREADS>::kRow, kRuns = Lanes<F, THREADS>::kRuns, kSteps = kRuns * L;
    static_assert(kSteps == kGateStateSteps, "a tile starts from a state that was kept");
    static_assert(L <= kRow && L < 32, "flags: a lane per step");
    __shared__ uint32_t s_tile;
    __shared__ float sU[kRuns][kGateCols], sH[kRuns][kGateCols], sC[kRuns][kGateCols];
    __shared__ float sPU[kRuns][kGateCols], sPC[kRuns][kGateCols];    // what comes behind them in the tile
    __shared__ float sCarry[kGateCols];
    __shared__ uint32_t sF[kRuns];

    const TileOf at = take_tile(p.tiles, &s_tile);
    const int64_t tile = p.tiles.nt - 1 - at.tile;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, q = tid & (kRow - 1), run = tid / kRow;
    const int64_t b = at.chain / p.tiles.nfb, fb = at.chain - b * p.tiles.nfb;
    const int64_t slot = at.tile * p.tiles.nchains + at.chain;
    const int64_t row0 = tile * kSteps, rows = p.T - row0, tape0 = b * p.T + row0;
    const int64_t f0 = fb * kGateCols + F * q;
    const int left = p.d - f0 >= F ? F : p.d > f0 ? (int)(p.d - f0) : 0;
    constexpr int S = Few<BF16, F>::SIZE, W = Few<BF16, F>::WORDS;
    const int64_t line = p.d * S;

    const Rsrc rs_st = make_rsrc(p.start + tape0, rows);
    const uint32_t flag = q < L ? bload_u8(rs_st, (uint32_t)(run * L + q)) : 0u;
    const Rsrc rs_x = make_rsrc((const char*)p.x + tape0 * line, rows * line);
    const Rsrc rs_h = make_rsrc((const char*)p.g + tape0 * line, rows * line);
    const Rsrc rs_g = make_rsrc((const char*)p.gates + 2 * tape0 * line, 2 * rows * line);
    const uint32_t off = left ? (uint32_t)(run * L * line + f0 * S) : kOob, step = left ? (uint32_t)line : 0u;
    const uint32_t goff = left ? (uint32_t)(2 * run * L * line + f0 * S) : kOob;
    Few<BF16, F> x[L], r[L], i[L], g[L];
#pragma unroll
    for (int s = 0; s < L; ++s) {
        r[s].template load<0, FULL>(rs_g, goff + 2 * s * step, left);
        i[s].template load<0, FULL>(rs_g, goff + (2 * s + 1) * step, left);
        x[s].template load<0, FULL>(rs_x, off + s * step, left);
        g[s].template load<0, FULL>(rs_h, off + s * step, left);
    }
    float rate[F], most = 0.0f;
#pragma unroll
    for (int e = 0; e < F; ++e) {
        rate[e] = e < left ? __builtin_fabsf(p.alpha[f0 + e]) : 0.0f;
        most = __builtin_fmaxf(most, rate[e]);
    }
    __builtin_amdgcn_sched_barrier(0);
    const uint64_t flags = __ballot(flag != 0u);
    const uint32_t begins = (uint32_t)(flags >> (lane & (64 - kRow))) & ((1u << L) - 1u);
    const bool slow = __all(most <= kSlow);
    if (rows < kSteps) {
        // steps behind the tape leave h and c as they are: r = -inf
#pragma unroll
        for (int s = 0; s < L; ++s)
            if (run * L + s >= rows) {
#pragma unroll
                for (int e = 0; e < W; ++e) r[s].w[e] = BF16 ? 0xFF80FF80u : 0xFF800000u;
            }
    }

    // ---- the runs' effects on h, forwards, and on c, backwards
    float k[L][F], sr[L][F], si[L][F], u[F] = {}, h[F] = {}, c[F] = {};
    using Yes = std::true_type;
    using No = std::false_type;
    auto effects = [&](auto SLOW, auto BEGINS) {
#pragma unroll
        for (int s = 0; s < L; ++s) {
            r[s].opaque();
            i[s].opaque();
            x[s].opaque();
            g[s].opaque();
#pragma unroll
            for (int e = 0; e < F; ++e) {
                const Gate<BF16, SLOW.value> gate(r[s].get(e), i[s].get(e), rate[e]);
                k[s][e] = gate.decay.k;
                sr[s][e] = gate.sr;
                si[s][e] = gate.si;
                u[e] += gate.u;
                const float v = gate.m * gate.si * x[s].get(e);
                const float next = gate.decay.of(h[e], v);
                h[e] = BEGINS.value && (begins >> s & 1u) ? v : next;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int s = L - 1; s >= 0; --s)
#pragma unroll
            for (int e = 0; e < F; ++e) {
                Decay<SLOW.value> d;
                d.k = k[s][e];
                const float next = d.of(g[s].get(e) + c[e]);
                c[e] = BEGINS.value && (begins >> s & 1u) ? 0.0f : next;
            }
    };
    if (slow) {
        if (flags) effects(Yes{}, Yes{});
        else effects(Yes{}, No{});
    } else {
        effects(No{}, Yes{});
    }
#pragma unroll
    for (int e = 0; e < F; ++e) {
        sU[run][F * q + e] = u[e];
        sH[run][F * q + e] = h[e];
        sC[run][F * q + e] = c[e];
    }
    if (q == 0) sF[run] = begins != 0u;
    barrier_lds();

    // ---- one behind the other, a lane per feature
    uint32_t held = 0;                                               // runs with a begin step
    if (lane < kRuns) held = sF[lane];
    held = (uint32_t)__ballot(held != 0u && lane < kRuns);
    float tu = 0.0f, tc = 0.0f;
    const bool in = fb * kGateCols + lane < p.d;
    const int64_t f = fb * kGateCols + lane;
    if (wave < 2) {
#pragma unroll
        for (int n = kRuns - 1; n >= 0; --n) {
            if (wave == 0) {
                sPU[n][lane] = tu;
                sPC[n][lane] = tc;
            }
            const float nu = sU[n][lane], nc = sC[n][lane];
            const float next = Decay<false>(nu).of(tc, nc);
            tc = held >> n & 1u ? nc : next;
            tu += nu;
        }
        const float first = at.tile == 0 && p.grad_state && in ? p.grad_state[b * p.d + f] : 0.0f;
        if (wave == 1) {
            if (p.tiles.nt > 1 && in) {
                if (held) put_incl(p.tiles, slot, lane, tc);
                else if (at.tile == 0) put_incl(p.tiles, slot, lane, Decay<false>(tu).of(first, tc));
                else put_agg(p.tiles, slot, lane, tu, tc);
            }
        } else {
            sCarry[lane] = at.tile == 0 ? first : look_back(p.tiles, at.tile, at.chain, lane, in);
        }
    } else if (wave == 2) {
        // (in place: the state that enters a run for what the run does to one)
        float now = in ? p.states[(b * p.tiles.nt + tile) * p.d + f] : 0.0f;
#pragma unroll
        for (int n = 0; n < kRuns; ++n) {
            const float nh = sH[n][lane];
            sH[n][lane] = now;
            const float next = Decay<false>(sU[n][lane]).of(now, nh);
            now = held >> n & 1u ? nh : next;
        }
    }
    barrier_lds();

    // ---- h before every step; then back with c
    if (wave == 1 && p.tiles.nt > 1 && at.tile > 0 && !held && in)
        put_incl(p.tiles, slot, lane, Decay<false>(tu).of(sCarry[lane], tc));
    const bool cut = held >> run >> 1 != 0u;                         // a begin step behind this run
    float sum[F] = {};
#pragma unroll
    for (int e = 0; e < F; ++e) {
        h[e] = sH[run][F * q + e];
        const float pc = sPC[run][F * q + e];
        const float from = Decay<false>(sPU[run][F * q + e]).of(sCarry[F * q + e], pc);
        c[e] = cut ? pc : from;
    }
    const Rsrc rs_dx = make_rsrc((char*)p.dx + tape0 * line, rows * line);
    const Rsrc rs_dg = make_rsrc((char*)p.dgates + 2 * tape0 * line, 2 * rows * line);
    uint32_t out = off, gout = goff;
    asm volatile("" : "+v"(out), "+v"(gout));                        // (the loads' offsets need not be kept for this)
    out += (L - 1) * step;
    gout += 2 * (L - 1) * step;
    auto back = [&](auto SLOW, auto BEGINS) {
        float before[L][F];
#pragma unroll
        for (int s = 0; s < L; ++s) {
            x[s].opaque();
            g[s].opaque();
#pragma unroll
            for (int e = 0; e < F; ++e) {
                const bool begin = BEGINS.value && (begins >> s & 1u);
                Decay<SLOW.value> d;
                d.k = k[s][e];
                const float w = d.taken();
                const float v = __builtin_amdgcn_sqrtf(w * (2.0f - w)) * si[s][e] * x[s].get(e);
                const float next = d.of(h[e], v);
                before[s][e] = begin ? 0.0f : h[e];
                h[e] = begin ? v : next;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int s = L - 1; s >= 0; --s) {
            // (what the loop above has formed of these is formed again rather than kept)
            x[s].opaque();
#pragma unroll
            for (int e = 0; e < F; ++e) asm volatile("" : "+v"(k[s][e]), "+v"(si[s][e]), "+v"(sr[s][e]));
            float dx[F], dr[F], di[F];
#pragma unroll
            for (int e = 0; e < F; ++e) {
                Decay<SLOW.value> d;
                d.k = k[s][e];
                const float w = d.taken(), a = d.left(), m2 = w * (2.0f - w);
                // (where nothing decays, m = 0 and 1 / m is to stay finite)
                const float rm = __builtin_amdgcn_rsqf(__builtin_fmaxf(m2, 0x1p-100f));
                const float xs = x[s].get(e) * si[s][e], m = m2 * rm;
                const float lam = g[s].get(e) + c[e];
                const float du = lam * a * __builtin_fmaf(xs * a, rm, -before[s][e]);
                const float ds = du * sr[s][e];
                sum[e] += ds;
                dx[e] = lam * m * si[s][e];
                dr[e] = ds * rate[e] * (1.0f - sr[s][e]);
                di[e] = lam * m * xs * (1.0f - si[s][e]);
                const float next = d.of(lam);
                c[e] = BEGINS.value && (begins >> s & 1u) ? 0.0f : next;
            }
            Few<BF16, F> o;
            o.set(dx);
            o.template store<kNt, FULL>(rs_dx, out, left);
            o.set(dr);
            o.template store<kNt, FULL>(rs_dg, gout, left);
            o.set(di);
            o.template store<kNt, FULL>(rs_dg, gout + step, left);
            out -= step;
            gout -= 2 * step;
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (slow) {
        if (flags) back(Yes{}, Yes{});
        else back(Yes{}, No{});
    } else {
        back(No{}, Yes{});
    }
    if (tile == 0 && run == 0 && p.grad_state_in) {
#pragma unroll
        for (int e = 0; e < F; ++e)
            if (e < left) p.grad_state_in[b * p.d + f0 + e] = c[e];
    }
    if (!p.part) return;
    // (nobody reads sU any more: its last readers passed the barrier above)
#pragma unroll
    for (int e = 0; e < F; ++e) sU[run][F * q + e] = sum[e];
    barrier_lds();
    if (wave == 0 && in) {
        float t = 0.0f;
#pragma unroll
        for (int n = 0; n < kRuns; ++n) t += sU[n][lane];
        p.part[(tile * p.B + b) * p.d + f] = t;
    }
}

// dalpha from the rows of partial sums: 64 features and 16 rows at a time
__global__ __launch_bounds__(1024) void gated_alpha_kernel(const float* part, const float* alpha, float* dalpha,
                                                           int64_t rows, int64_t d) {
    __shared__ double s[16][64];
    const int col = threadIdx.x & 63, row = threadIdx.x >> 6;
    const int64_t f = (int64_t)blockIdx.x * 64 + col;
    double sum = 0.0;
    if (f < d)
        for (int64_t r = row; r < rows; r += 16) sum += (double)part[r * d + f];
    s[row][col] = sum;
    __syncthreads();
    if (row == 0 && f < d) {
        for (int r = 1; r < 16; ++r) sum += s[r][col];
        const float a = alpha[f];
        dalpha[f] = a > 0.0f ? (float)sum : a < 0.0f ? (float)-sum : 0.0f;
    }
}

template <bool BF16, bool FULL>
void bwd(const GatedBwdArgs& a, hipStream_t s) {
    constexpr GateShape sh = gate_bwd_shape(BF16);
    hipLaunchKernelGGL((gated_bwd_kernel<BF16, FULL, sh.f, sh.steps, sh.threads, sh.waves>),
                       dim3((unsigned)(a.tiles.nt * a.tiles.nchains)), dim3(sh.threads), 0, s, a);
}

}  // namespace

hipError_t gated_bwd_launch(bool bf16, bool full, const GatedBwdArgs& a, hipStream_t s) {
    if (bf16) full ? bwd<true, true>(a, s) : bwd<true, false>(a, s);
    else full ? bwd<false, true>(a, s) : bwd<false, false>(a, s);
    if (!a.part) return hipGetLastError();
    hipLaunchKernelGGL(gated_alpha_kernel, dim3((unsigned)((a.d + 63) / 64)), dim3(1024), 0, s, a.part, a.alpha, a.dalpha,
                       a.part_rows, a.d);
    return hipGetLastError();
}

}  // namespace memoroid
