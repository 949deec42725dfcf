// gated_fwd.hip -- the gated recurrence, forward, in one pass over memory.
//
// A tile is 16 runs of L steps of 64 features (gated_common.hpp).  (1) All loads of a lane
// go out first; (2) the gates of its L steps give decays and inputs, kept in registers, and
// the run's effect on a state: its rates' sum and what it adds; (3) one wavefront puts
// the runs' effects one behind the other through LDS while another publishes the
// tile's; (4) the first looks back for the state that enters the tile; (5) every lane runs
// its steps from the state that enters them and stores h.  Gates are formed once: with
// six transcendental instructions and some thirty others a value, bf16 is nearly as much
// instruction issue as memory traffic.
#include <type_traits>

#include "gated_common.hpp"

namespace memoroid {

namespace {

template <bool BF16, bool FULL, int F, int L, int THREADS, int WAVES>
__global__ __launch_bounds__(THREADS, WAVES) void gated_fwd_kernel(GatedFwdArgs p) {
    constexpr int kRow = Lanes<F, THREADS>::kRow, kRuns = Lanes<F, THREADS>::kRuns, kSteps = kRuns * L;
    static_assert(L <= kRow && L < 32 && kGateStateSteps % L == 0, "flags: a lane per step; states lie between runs");
    __shared__ uint32_t s_tile;
    __shared__ float sU[kRuns][kGateCols], sH[kRuns][kGateCols];      // runs: rates' sum, added
    __shared__ float sPU[kRuns][kGateCols], sPH[kRuns][kGateCols];    // what comes before them in the tile
    __shared__ float sCarry[kGateCols];
    __shared__ uint32_t sF[kRuns];

    const TileOf at = take_tile(p.tiles, &s_tile);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, q = tid & (kRow - 1), run = tid / kRow;
    const int64_t b = at.chain / p.tiles.nfb, fb = at.chain - b * p.tiles.nfb;
    const int64_t slot = at.tile * p.tiles.nchains + at.chain;
    const int64_t row0 = at.tile * kSteps, rows = p.T - row0, tape0 = b * p.T + row0;
    const int64_t f0 = fb * kGateCols + F * q;
    const int left = p.d - f0 >= F ? F : p.d > f0 ? (int)(p.d - f0) : 0;
    constexpr int S = Few<BF16, F>::SIZE;
    const int64_t line = p.d * S;                                    // bytes of a row of x

    // ---- (1)
    const Rsrc rs_st = make_rsrc(p.start + tape0, rows);
    const uint32_t flag = q < L ? bload_u8(rs_st, (uint32_t)(run * L + q)) : 0u;
    const Rsrc rs_x = make_rsrc((const char*)p.x + tape0 * line, rows * line);
    const Rsrc rs_g = make_rsrc((const char*)p.gates + 2 * tape0 * line, 2 * rows * line);
    const uint32_t off = left ? (uint32_t)(run * L * line + f0 * S) : kOob, step = left ? (uint32_t)line : 0u;
    const uint32_t goff = left ? (uint32_t)(2 * run * L * line + f0 * S) : kOob;
    Few<BF16, F> x[L], r[L], i[L];
#pragma unroll
    for (int s = 0; s < L; ++s) {
        r[s].template load<0, FULL>(rs_g, goff + 2 * s * step, left);
        i[s].template load<0, FULL>(rs_g, goff + (2 * s + 1) * step, left);
        x[s].template load<0, FULL>(rs_x, off + s * step, left);
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

    // ---- (2)
    float k[L][F], v[L][F], u[F] = {}, h[F] = {};
    auto gates = [&](auto SLOW) {
#pragma unroll
        for (int s = 0; s < L; ++s) {
            // (keeps the two branches' common work, all steps' of it, from being done ahead of
            // the branch, in registers that are not there)
            r[s].opaque();
            i[s].opaque();
            x[s].opaque();
#pragma unroll
            for (int e = 0; e < F; ++e) {
                const Gate<BF16, SLOW.value> g(r[s].get(e), i[s].get(e), rate[e]);
                k[s][e] = g.decay.k;
                v[s][e] = g.m * g.si * x[s].get(e);
                u[e] += g.u;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // a state through the run; `each` sees it after every step
    auto through = [&](auto SLOW, auto BEGINS, auto each) {
#pragma unroll
        for (int s = 0; s < L; ++s) {
#pragma unroll
            for (int e = 0; e < F; ++e) {
                Decay<SLOW.value> d;
                d.k = k[s][e];
                const float next = d.of(h[e], v[s][e]);
                h[e] = BEGINS.value && (begins >> s & 1u) ? v[s][e] : next;
            }
            each(s);
        }
    };
    using Yes = std::true_type;
    using No = std::false_type;
    auto run_through = [&](auto each) {
        if (slow) {
            if (flags) through(Yes{}, Yes{}, each);
            else through(Yes{}, No{}, each);
        } else {
            through(No{}, Yes{}, each);
        }
    };
    if (slow) gates(Yes{});
    else gates(No{});
    run_through([](int) {});
#pragma unroll
    for (int e = 0; e < F; ++e) {
        sU[run][F * q + e] = u[e];
        sH[run][F * q + e] = h[e];
    }
    if (q == 0) sF[run] = begins != 0u;
    barrier_lds();

    // ---- (3), (4): a lane per feature
    uint32_t held = 0;                                               // runs with a begin step
    if (lane < kRuns) held = sF[lane];
    held = (uint32_t)__ballot(held != 0u && lane < kRuns);
    float tu = 0.0f, th = 0.0f;
    const bool in = fb * kGateCols + lane < p.d;
    if (wave < 2) {
#pragma unroll
        for (int g = 0; g < kRuns; ++g) {
            if (wave == 0) {
                sPU[g][lane] = tu;
                sPH[g][lane] = th;
            }
            const float gu = sU[g][lane], gh = sH[g][lane];
            const float next = Decay<false>(gu).of(th, gh);
            th = held >> g & 1u ? gh : next;
            tu += gu;
        }
        const float first = at.tile == 0 && p.state_in && in ? p.state_in[b * p.d + fb * kGateCols + lane] : 0.0f;
        if (wave == 1) {
            if (p.tiles.nt > 1 && in) {
                if (held) put_incl(p.tiles, slot, lane, th);
                else if (at.tile == 0) put_incl(p.tiles, slot, lane, Decay<false>(tu).of(first, th));
                else put_agg(p.tiles, slot, lane, tu, th);
            }
        } else {
            const bool first_begins = flags & 1u;                    // (this wavefront's first lane: the tile's first step)
            sCarry[lane] = at.tile == 0 ? first : look_back(p.tiles, at.tile, at.chain, lane, in && !first_begins);
            if (at.tile == 0 && p.states && in)
                p.states[b * ((p.T + kGateStateSteps - 1) / kGateStateSteps) * p.d + fb * kGateCols + lane] = first;
        }
    }
    barrier_lds();

    // ---- (5)
    if (wave == 1 && p.tiles.nt > 1 && at.tile > 0 && !held && in)
        put_incl(p.tiles, slot, lane, Decay<false>(tu).of(sCarry[lane], th));
    const bool cut = (held & ((1u << run) - 1u)) != 0u;              // a begin step before this run
#pragma unroll
    for (int e = 0; e < F; ++e) {
        const float ph = sPH[run][F * q + e];
        const float from = Decay<false>(sPU[run][F * q + e]).of(sCarry[F * q + e], ph);
        h[e] = cut ? ph : from;
    }
    const Rsrc rs_h = make_rsrc((char*)p.h + tape0 * line, rows * line);
    uint32_t out = off;
    asm volatile("" : "+v"(out));                                    // (the loads' offsets need not be kept for this)
    const int64_t last = rows - 1 - (int64_t)run * L;                // the tape's last step, seen from this run
    run_through([&](int s) {
        Few<BF16, F> o;
        o.set(h);
        o.template store<kNt, FULL>(rs_h, out, left);
        out += step;
        if (s == last && p.state_out) {
#pragma unroll
            for (int e = 0; e < F; ++e)
                if (e < left) p.state_out[b * p.d + f0 + e] = h[e];
        }
    });
    const int64_t next = row0 + (int64_t)(run + 1) * L;              // the step behind this run
    if (p.states && next % kGateStateSteps == 0 && next < p.T) {
        float* const o = p.states + (b * ((p.T + kGateStateSteps - 1) / kGateStateSteps) + next / kGateStateSteps) * p.d;
#pragma unroll
        for (int e = 0; e < F; ++e)
            if (e < left) o[f0 + e] = h[e];
    }
}

template <bool BF16, bool FULL>
void fwd(const GatedFwdArgs& a, hipStream_t s) {
    constexpr GateShape sh = gate_fwd_shape(BF16);
    hipLaunchKernelGGL((gated_fwd_kernel<BF16, FULL, sh.f, sh.steps, sh.threads, sh.waves>),
                       dim3((unsigned)(a.tiles.nt * a.tiles.nchains)), dim3(sh.threads), 0, s, a);
}

}  // namespace

hipError_t gated_fwd_launch(bool bf16, bool full, const GatedFwdArgs& a, hipStream_t s) {
    if (bf16) full ? fwd<true, true>(a, s) : fwd<true, false>(a, s);
    else full ? fwd<false, true>(a, s) : fwd<false, false>(a, s);
    return hipGetLastError();
}

}  // namespace memoroid
