// gated_bwd.hip -- gradient of the gated recurrence, in one pass over memory.
//
// With g = dL/dh and lam = dL/dh with what later steps add,
//     lam_t = g_t + c_t,   c_{t-1} = a_t lam_t  (0 at a begin step; the last c: dL/dstate),
//     dx = lam m sig(i),   di = lam b (1 - sig(i)),
//     du = lam a (sig(i) x a / m - h_before),   dr = du u (1 - sig(r)),
//     dalpha = sign(alpha) sum du sig(r).
// The forward call has kept the state before every tile (and more), so h is run through
// again within a tile and only c goes from tile to tile, the last first.  Otherwise
// as forward (gated_fwd.hip): the runs' effects on h and on c, put one behind the other
// by a wavefront each; then h through each run; then, with the c that enters, back through
// it, forming every gradient.  Sums for dalpha: a row per tile, added up by a second
// kernel in doubles.
//
// Seven tensors are read or written once: 8 tapes of 4096 steps of 2048 bf16 features, 0.94
// GB in 205 us, 4.6 TB/s, the VALU busy for 130 of them (67 instructions a value); fp32, 8 x
// 4096 x 1024, 190 us.  A step's coefficients that do not wait for the carry (m sig(i), v (1 -
// sig(i)), sig(i) x a / m) are formed before it comes: 264 -> 234 us beside forming all gates
// twice.  The registers (five floats a step and feature) set the tile: 16 steps a lane leave room
// for two workgroups on a CU and take 238 us, 4 steps of 512 threads 271, and under 128 registers
// they spill.
#include <type_traits>

#include "gated_common.hpp"

namespace memoroid {

namespace {

template <bool BF16, bool FULL, int POL, int L, int THREADS, int WAVES>
__global__ __launch_bounds__(THREADS, WAVES) void gated_bwd_kernel(GatedBwdArgs p) {
    constexpr int kLd = POL == kStreamAll ? kNt : 0, kSt = POL != kCached ? kNt : 0;
    constexpr int F = 2, kRow = Lanes<F, THREADS>::kRow, kRuns = Lanes<F, THREADS>::kRuns, kSteps = kRuns * L;
    static_assert(L <= kRow && L < 32, "flags: a lane per step");
    __shared__ uint32_t s_tile;
    // per run: its rates' sum, its decay, what it adds to h and to c (then the state that enters
    // it in the place of the one), the c that enters it
    __shared__ float sU[kRuns][kGateCols], sK[kRuns][kGateCols], sH[kRuns][kGateCols], sC[kRuns][kGateCols];
    __shared__ float sIn[kRuns][kGateCols];
    __shared__ LookBackLds sLook;
    __shared__ uint32_t sF[kRuns];

    const TileOf at = take_tile(p.tiles, &s_tile);
    const int64_t tile = p.tiles.nt - 1 - at.tile;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, q = tid & (kRow - 1), run = tid / kRow;
    const int64_t b = at.chain / p.tiles.nfb, fb = at.chain - b * p.tiles.nfb;
    const int64_t slot = at.tile * p.tiles.nchains + at.chain;
    const int64_t row0 = tile * kSteps, rows = p.T - row0, tape0 = b * p.T + row0;
    const int64_t f0 = fb * kGateCols + F * q;
    const int left = p.d - f0 >= F ? F : p.d > f0 ? (int)(p.d - f0) : 0;
    constexpr int S = Few<BF16>::SIZE, W = Few<BF16>::WORDS;
    const int64_t line = p.d * S;

    const Rsrc rs_st = make_rsrc(p.start + tape0, rows);
    const uint32_t flag = q < L ? bload_u8(rs_st, (uint32_t)(run * L + q)) : 0u;
    const Rows rs_x = rows_at((const char*)p.x + tape0 * line, rows * line);
    const Rows rs_h = rows_at((const char*)p.g + tape0 * line, rows * line);
    const Rows rs_g = rows_at((const char*)p.gates + 2 * tape0 * line, 2 * rows * line);
    const uint32_t off = left ? (uint32_t)(run * L * line + f0 * S) : kOob;
    const uint32_t goff = left ? (uint32_t)(2 * run * L * line + f0 * S) : kOob;
    const uint32_t step = (uint32_t)line;
    // (a whole tile's rows by scalar offsets, the last tile's by the lanes': gated_fwd.hip)
    const bool whole = rows >= kSteps, wide = p.d > 1;
    Few<BF16> x[L], r[L], i[L], g[L];
    if (whole) {
#pragma unroll
        for (int s = 0; s < L; ++s) {
            r[s].template load<kLd, FULL>(rs_g, goff, 2 * s * step, left, true, wide);
            i[s].template load<kLd, FULL>(rs_g, goff, (2 * s + 1) * step, left, true, wide);
            x[s].template load<kLd, FULL>(rs_x, off, s * step, left, true, wide);
            g[s].template load<kLd, FULL>(rs_h, off, s * step, left, true, wide);
        }
    } else {
        const uint32_t by = left ? step : 0u;
#pragma unroll
        for (int s = 0; s < L; ++s) {
            r[s].template load<kLd, FULL>(rs_g, goff + 2 * s * by, 0, left, run * L + s < rows, wide);
            i[s].template load<kLd, FULL>(rs_g, goff + (2 * s + 1) * by, 0, left, run * L + s < rows, wide);
            x[s].template load<kLd, FULL>(rs_x, off + s * by, 0, left, run * L + s < rows, wide);
            g[s].template load<kLd, FULL>(rs_h, off + s * by, 0, left, run * L + s < rows, wide);
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
    // Kept of a step, for the way back: the decay k, sig(r), and of what does not wait for h
    // and c dx / lam, di / lam and sig(i) x a / m less the run's own h before the step
    float k[L][F], sr[L][F], px[L][F], pi[L][F], z[L][F];
    float u[F] = {}, h[F] = {}, c[F] = {};
    using Yes = std::true_type;
    using No = std::false_type;
    auto effects = [&](auto SLOW, auto BEGINS) {
#pragma unroll
        for (int s = 0; s < L; ++s) {
            r[s].opaque();
            i[s].opaque();
            x[s].opaque();
            g[s].opaque();
            r[s].template settle<FULL>(left, wide);
            i[s].template settle<FULL>(left, wide);
            x[s].template settle<FULL>(left, wide);
            g[s].template settle<FULL>(left, wide);
#pragma unroll
            for (int e = 0; e < F; ++e) {
                const float gr = sigmoid<BF16>(r[s].get(e)), gi = sigmoid<BF16>(i[s].get(e)), gu = rate[e] * gr;
                const Decay<SLOW.value, BF16> d(gu);
                const float w = d.taken(), m2 = w * (2.0f - w);
                // (where nothing decays, m = 0: no 1 / m, and the term that has it none either; the
                // root forward has no normal result there)
                const float rm = m2 >= 0x1p-126f ? __builtin_amdgcn_rsqf(m2) : 0.0f, m = m2 * rm;
                const float xs = x[s].get(e) * gi, v = m * xs;
                const bool begin = BEGINS.value && (begins >> s & 1u);
                k[s][e] = d.k;
                sr[s][e] = gr;
                px[s][e] = m * gi;
                pi[s][e] = __builtin_fmaf(-v, gi, v);
                z[s][e] = xs * rm * d.left() - (begin ? 0.0f : h[e]);
                u[e] += gu;
                const float next = d.of(h[e], v);
                h[e] = begin ? v : next;
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
        sK[run][F * q + e] = Decay<false>(u[e]).k;
        sH[run][F * q + e] = h[e];
        sC[run][F * q + e] = c[e];
    }
    if (q == 0) sF[run] = begins != 0u;
    barrier_lds();

    // ---- one behind the other, a lane per feature
    uint32_t held = 0;                                               // runs with a begin step
    if (lane < kRuns) held = sF[lane];
    held = (uint32_t)__ballot(held != 0u && lane < kRuns);
    const bool in = fb * kGateCols + lane < p.d;
    const int64_t f = fb * kGateCols + lane;
    auto apply = [&](int n, float v, float add) {
        Decay<false> d;
        d.k = sK[n][lane];
        const float next = d.of(v, add);
        return held >> n & 1u ? add : next;
    };
    // (wavefronts 0 and 1: the tile's own effect, as forward)
    float tc = 0.0f;
    Decay<false> all;
    if (wave < 2 && p.tiles.nt > 1) {
        float u = 0.0f;
#pragma unroll
        for (int n = kRuns - 1; n >= 0; --n) {
            tc = apply(n, tc, sC[n][lane]);
            u += sU[n][lane];
        }
        all = Decay<false>(u);
    }
    const float first = wave < 2 && at.tile == 0 && p.grad_state && in ? p.grad_state[b * p.d + f] : 0.0f;
    auto enter = [&](float v) {
        if (at.tile > 0 && in && !held) put_incl(p.tiles, slot, lane, all.of(v, tc));
#pragma unroll
        for (int n = kRuns - 1; n >= 0; --n) {
            sIn[n][lane] = v;
            v = apply(n, v, sC[n][lane]);
        }
    };
    if (wave == 0) {
        float v = first;
        const bool there = at.tile == 0 || try_near(p.tiles, at.tile, at.chain, lane, in, v);
        if (there) enter(v);
        if (lane == 0) sLook.done = there;
    } else if (wave == 1) {
        if (p.tiles.nt > 1 && in) {
            if (held) put_incl(p.tiles, slot, lane, tc);
            else if (at.tile == 0) put_incl(p.tiles, slot, lane, all.of(first, tc));
            else put_agg(p.tiles, slot, lane, all.k, tc);
        }
    } else if (wave == 2) {
        const int64_t ns = (p.T + kGateStateSteps - 1) / kGateStateSteps;
        float v = in ? p.states[(b * ns + tile * kSteps / kGateStateSteps) * p.d + f] : 0.0f;
#pragma unroll
        for (int n = 0; n < kRuns; ++n) {
            const float add = sH[n][lane];
            sH[n][lane] = v;
            v = apply(n, v, add);
        }
    }
    barrier_lds();
    if (!sLook.done) look_far<THREADS, BF16 ? 4 : 8>(p.tiles, at.tile, at.chain, lane, in, sLook, enter);

    // ---- the state that enters the run goes into z; then back with c
    float sum[F] = {};
#pragma unroll
    for (int e = 0; e < F; ++e) {
        h[e] = sH[run][F * q + e];
        c[e] = sIn[run][F * q + e];
    }
    const Rows rs_dx = rows_at((char*)p.dx + tape0 * line, rows * line);
    const Rows rs_dg = rows_at((char*)p.dgates + 2 * tape0 * line, 2 * rows * line);
    auto back = [&](auto SLOW, auto BEGINS) {
        // (h: what is left of the entering state before each step)
#pragma unroll
        for (int s = 0; s < L; ++s)
#pragma unroll
            for (int e = 0; e < F; ++e) {
                Decay<SLOW.value> d;
                d.k = k[s][e];
                const bool begin = BEGINS.value && (begins >> s & 1u);
                z[s][e] -= begin ? 0.0f : h[e];
                h[e] = begin ? 0.0f : d.of(h[e]);
            }
#pragma unroll
        for (int s = L - 1; s >= 0; --s) {
            g[s].opaque();
            float dx[F], dr[F], di[F];
#pragma unroll
            for (int e = 0; e < F; ++e) {
                Decay<SLOW.value> d;
                d.k = k[s][e];
                const float lam = g[s].get(e) + c[e];
                const float next = d.of(lam), ds = next * z[s][e] * sr[s][e], du = ds * rate[e];
                sum[e] += ds;
                dx[e] = lam * px[s][e];
                dr[e] = __builtin_fmaf(-du, sr[s][e], du);
                di[e] = lam * pi[s][e];
                c[e] = BEGINS.value && (begins >> s & 1u) ? 0.0f : next;
            }
            Few<BF16> o;
            const uint32_t by = whole || !left ? 0u : step, sby = whole ? step : 0u;
            const bool in_tape = whole || run * L + s < rows;
            o.set(dx);
            o.template store<kSt, FULL>(rs_dx, off + s * by, s * sby, left, in_tape);
            o.set(dr);
            o.template store<kSt, FULL>(rs_dg, goff + 2 * s * by, 2 * s * sby, left, in_tape);
            o.set(di);
            o.template store<kSt, FULL>(rs_dg, goff + (2 * s + 1) * by, (2 * s + 1) * sby, left, in_tape);
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

// dalpha from the rows of partial sums, in doubles: 32 features, 32 rows at a time
__global__ __launch_bounds__(1024) void gated_alpha_kernel(const float* part, const float* alpha, float* dalpha,
                                                           int64_t rows, int64_t d) {
    __shared__ double s[32][32];
    const int col = threadIdx.x & 31, row = threadIdx.x >> 5;
    const int64_t f = (int64_t)blockIdx.x * 32 + col;
    double sum = 0.0;
    if (f < d) {
#pragma unroll 8
        for (int64_t r = row; r < rows; r += 32) sum += (double)part[r * d + f];
    }
    s[row][col] = sum;
    __syncthreads();
    if (row == 0 && f < d) {
        for (int r = 1; r < 32; ++r) sum += s[r][col];
        const float a = alpha[f];
        dalpha[f] = a > 0.0f ? (float)sum : a < 0.0f ? (float)-sum : 0.0f;
    }
}

template <bool BF16, bool FULL, int POL, int UPTO>
void launch_for(const GatedBwdArgs& a, hipStream_t s) {
    constexpr GateShape sh = gate_bwd_shape(BF16, UPTO);
    static_assert(sh.tile() % kGateStateSteps == 0 || UPTO <= sh.tile(), "a tile starts from a state that was kept");
    hipLaunchKernelGGL((gated_bwd_kernel<BF16, FULL, POL, sh.steps, sh.threads, sh.waves>),
                       dim3((unsigned)(a.tiles.nt * a.tiles.nchains)), dim3(sh.threads), 0, s, a);
}
template <bool BF16, bool FULL, int POL>
void launch(const GatedBwdArgs& a, hipStream_t s) {
    if (a.T <= 32) launch_for<BF16, FULL, POL, 32>(a, s);
    else launch_for<BF16, FULL, POL, 33>(a, s);
}
// (rows that lanes cannot take whole are not whole lines either)
template <bool BF16>
void with_policy(bool full, int policy, const GatedBwdArgs& a, hipStream_t s) {
    if (!full) launch<BF16, false, kCached>(a, s);
    else if (policy == kCached) launch<BF16, true, kCached>(a, s);
    else if (policy == kStreamOut) launch<BF16, true, kStreamOut>(a, s);
    else launch<BF16, true, kStreamAll>(a, s);
}

}  // namespace

hipError_t gated_bwd_launch(bool bf16, bool full, int policy, const GatedBwdArgs& a, hipStream_t s) {
    bf16 ? with_policy<true>(full, policy, a, s) : with_policy<false>(full, policy, a, s);
    if (!a.part) return hipGetLastError();
    hipLaunchKernelGGL(gated_alpha_kernel, dim3((unsigned)((a.d + 31) / 32)), dim3(1024), 0, s, a.part, a.alpha, a.dalpha,
                       a.part_rows, a.d);
    return hipGetLastError();
}

}  // namespace memoroid
