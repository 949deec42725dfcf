// gated_fwd.hip -- the gated recurrence, forward, in one pass over memory.
//
// A tile is 8 runs of L steps of 64 features (gated_common.hpp).  (1) All loads of a lane
// go out first; (2) the gates of its L steps give decays and inputs, kept in registers, and
// the run's effect on a state: its rates' sum and what it adds; (3) one wavefront puts
// the runs' effects one behind the other through LDS while another publishes the
// tile's; (4) the first looks back for the state that enters the tile; (5) every lane runs
// its steps from the state that enters them and stores h.
//
// Memory bounds it, with instruction issue close behind.  8 tapes of 4096 steps of 2048
// bf16 features: 0.54 GB in 112 us, 4.8 TB/s (a copy of 2 GiB reaches 4.9, a pass that
// reads as much as it writes 6.1), of which the VALU is busy for 72: 35 instructions a value, six
// of them transcendental in two issue slots, so gates are formed once and decays stay in
// registers.  Without the look-back it takes 5 us less, without the gates' arithmetic another
// 4, so what is left is the loads of a workgroup, which all go out at its start.  fp32, 8 x 4096 x
// 1024: 110 us, 4.9 TB/s.  T = 65536 x 2048, where 32 chains are 512 tiles long: 221 us, 35 of
// them for the look-back.
#include <type_traits>

#include "gated_common.hpp"

namespace memoroid {

namespace {

template <bool BF16, bool FULL, int POL, int L, int THREADS, int WAVES>
__global__ __launch_bounds__(THREADS, WAVES) void gated_fwd_kernel(GatedFwdArgs p) {
    constexpr int kLd = POL == kStreamAll ? kNt : 0, kSt = POL != kCached ? kNt : 0;
    constexpr int F = 2, kRow = Lanes<F, THREADS>::kRow, kRuns = Lanes<F, THREADS>::kRuns, kSteps = kRuns * L;
    static_assert(L <= kRow && L < 32 && kGateStateSteps % L == 0, "flags: a lane per step; states lie between runs");
    __shared__ uint32_t s_tile;
    // per run: its rates' sum, its decay, what it adds, the state that enters it
    __shared__ float sU[kRuns][kGateCols], sK[kRuns][kGateCols], sH[kRuns][kGateCols], sIn[kRuns][kGateCols];
    __shared__ LookBackLds sLook;
    __shared__ uint32_t sF[kRuns], sBegins;

    const TileOf at = take_tile(p.tiles, &s_tile);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, q = tid & (kRow - 1), run = tid / kRow;
    const int64_t b = at.chain / p.tiles.nfb, fb = at.chain - b * p.tiles.nfb;
    const int64_t slot = at.tile * p.tiles.nchains + at.chain;
    const int64_t row0 = at.tile * kSteps, rows = p.T - row0, tape0 = b * p.T + row0;
    const int64_t f0 = fb * kGateCols + F * q;
    const int left = p.d - f0 >= F ? F : p.d > f0 ? (int)(p.d - f0) : 0;
    constexpr int S = Few<BF16>::SIZE;
    const int64_t line = p.d * S;                                    // bytes of a row of x

    // ---- (1)
    const Rsrc rs_st = make_rsrc(p.start + tape0, rows);
    const uint32_t flag = q < L ? bload_u8(rs_st, (uint32_t)(run * L + q)) : 0u;
    const Rows rs_x = rows_at((const char*)p.x + tape0 * line, rows * line);
    const Rows rs_g = rows_at((const char*)p.gates + 2 * tape0 * line, 2 * rows * line);
    const uint32_t off = left ? (uint32_t)(run * L * line + f0 * S) : kOob;
    const uint32_t goff = left ? (uint32_t)(2 * run * L * line + f0 * S) : kOob;
    const uint32_t step = (uint32_t)line;
    // A whole tile's rows are reached by scalar offsets; those of the tape's last tile by
    // the lanes', which the range check covers (lanes past d stay outside either way)
    const bool whole = rows >= kSteps, wide = p.d > 1;
    Few<BF16> x[L], r[L], i[L];
    if (whole) {
#pragma unroll
        for (int s = 0; s < L; ++s) {
            r[s].template load<kLd, FULL>(rs_g, goff, 2 * s * step, left, true, wide);
            i[s].template load<kLd, FULL>(rs_g, goff, (2 * s + 1) * step, left, true, wide);
            x[s].template load<kLd, FULL>(rs_x, off, s * step, left, true, wide);
        }
    } else {
        const uint32_t by = left ? step : 0u;
#pragma unroll
        for (int s = 0; s < L; ++s) {
            r[s].template load<kLd, FULL>(rs_g, goff + 2 * s * by, 0, left, run * L + s < rows, wide);
            i[s].template load<kLd, FULL>(rs_g, goff + (2 * s + 1) * by, 0, left, run * L + s < rows, wide);
            x[s].template load<kLd, FULL>(rs_x, off + s * by, 0, left, run * L + s < rows, wide);
        }
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
            r[s].template settle<FULL>(left, wide);
            i[s].template settle<FULL>(left, wide);
            x[s].template settle<FULL>(left, wide);
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
        sK[run][F * q + e] = Decay<false>(u[e]).k;
        sH[run][F * q + e] = h[e];
    }
    if (q == 0) sF[run] = begins != 0u;
    if (tid == 0) sBegins = begins & 1u;
    barrier_lds();

    // ---- (3), (4): a lane per feature
    uint32_t held = 0;                                               // runs with a begin step
    if (lane < kRuns) held = sF[lane];
    held = (uint32_t)__ballot(held != 0u && lane < kRuns);
    const bool in = fb * kGateCols + lane < p.d;
    auto apply = [&](int n, float v) {
        Decay<false> d;
        d.k = sK[n][lane];
        const float add = sH[n][lane], next = d.of(v, add);
        return held >> n & 1u ? add : next;
    };
    // the tile's own effect: wavefront 1 publishes it, the first needs it to publish the state
    // after the tile the moment it has the one before
    float th = 0.0f;
    Decay<false> all;
    if (wave < 2 && p.tiles.nt > 1) {
        float u = 0.0f;
#pragma unroll
        for (int n = 0; n < kRuns; ++n) {
            th = apply(n, th);
            u += sU[n][lane];
        }
        all = Decay<false>(u);
    }
    const float first = wave < 2 && at.tile == 0 && p.state_in && in ? p.state_in[b * p.d + fb * kGateCols + lane] : 0.0f;
    const bool need = in && !sBegins;                                // a tile that begins an episode takes nothing
    auto enter = [&](float v) {
        if (at.tile > 0 && in && !held) put_incl(p.tiles, slot, lane, all.of(v, th));
#pragma unroll
        for (int n = 0; n < kRuns; ++n) {
            sIn[n][lane] = v;
            v = apply(n, v);
        }
    };
    if (wave == 0) {
        float v = first;
        if (at.tile == 0 && p.states && in)
            p.states[b * ((p.T + kGateStateSteps - 1) / kGateStateSteps) * p.d + fb * kGateCols + lane] = v;
        const bool there = at.tile == 0 || try_near(p.tiles, at.tile, at.chain, lane, need, v);
        if (there) enter(v);
        if (lane == 0) sLook.done = there;
    } else if (wave == 1 && p.tiles.nt > 1 && in) {
        if (held) put_incl(p.tiles, slot, lane, th);
        else if (at.tile == 0) put_incl(p.tiles, slot, lane, all.of(first, th));
        else put_agg(p.tiles, slot, lane, all.k, th);
    }
    barrier_lds();
    if (!sLook.done) look_far<THREADS, BF16 ? 4 : 8>(p.tiles, at.tile, at.chain, lane, need, sLook, enter);

    // ---- (5)
#pragma unroll
    for (int e = 0; e < F; ++e) h[e] = sIn[run][F * q + e];
    const Rows rs_h = rows_at((char*)p.h + tape0 * line, rows * line);
    float from[F];
#pragma unroll
    for (int e = 0; e < F; ++e) from[e] = h[e];
    if (whole) {
        run_through([&](int s) {
            Few<BF16> o;
            o.set(h);
            o.template store<kSt, FULL>(rs_h, off, s * step, left, true);
        });
    } else {
        const uint32_t by = left ? step : 0u;
        through(No{}, Yes{}, [&](int s) {
            Few<BF16> o;
            o.set(h);
            o.template store<kSt, FULL>(rs_h, off + s * by, 0, left, run * L + s < rows);
        });
    }
    const int64_t last = rows - 1 - (int64_t)run * L;                // the tape's last step, seen from this run
    if (p.state_out && last >= 0 && last < L) {
        float end[F];
#pragma unroll
        for (int e = 0; e < F; ++e) {
            end[e] = h[e];
            h[e] = from[e];
        }
        through(No{}, Yes{}, [&](int s) {
#pragma unroll
            for (int e = 0; e < F; ++e)
                if (s == last && e < left) p.state_out[b * p.d + f0 + e] = h[e];
        });
#pragma unroll
        for (int e = 0; e < F; ++e) h[e] = end[e];
    }
    const int64_t next = row0 + (int64_t)(run + 1) * L;              // the step behind this run
    if (p.states && next % kGateStateSteps == 0 && next < p.T) {
        float* const o = p.states + (b * ((p.T + kGateStateSteps - 1) / kGateStateSteps) + next / kGateStateSteps) * p.d;
#pragma unroll
        for (int e = 0; e < F; ++e)
            if (e < left) o[f0 + e] = h[e];
    }
}

template <bool BF16, bool FULL, int POL, int UPTO>
void launch_for(const GatedFwdArgs& a, hipStream_t s) {
    constexpr GateShape sh = gate_fwd_shape(BF16, UPTO);
    hipLaunchKernelGGL((gated_fwd_kernel<BF16, FULL, POL, sh.steps, sh.threads, sh.waves>),
                       dim3((unsigned)(a.tiles.nt * a.tiles.nchains)), dim3(sh.threads), 0, s, a);
}
template <bool BF16, bool FULL, int POL>
void launch(const GatedFwdArgs& a, hipStream_t s) {
    if (a.T <= 32) launch_for<BF16, FULL, POL, 32>(a, s);
    else if (a.T <= 64) launch_for<BF16, FULL, POL, 64>(a, s);
    else launch_for<BF16, FULL, POL, 65>(a, s);
}
// (rows that lanes cannot take whole are not whole lines either)
template <bool BF16>
void with_policy(bool full, int policy, const GatedFwdArgs& a, hipStream_t s) {
    if (!full) launch<BF16, false, kCached>(a, s);
    else if (policy == kCached) launch<BF16, true, kCached>(a, s);
    else if (policy == kStreamOut) launch<BF16, true, kStreamOut>(a, s);
    else launch<BF16, true, kStreamAll>(a, s);
}

}  // namespace

hipError_t gated_fwd_launch(bool bf16, bool full, int policy, const GatedFwdArgs& a, hipStream_t s) {
    bf16 ? with_policy<true>(full, policy, a, s) : with_policy<false>(full, policy, a, s);
    return hipGetLastError();
}

}  // namespace memoroid
