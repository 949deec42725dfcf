// gated_common.hpp -- arithmetic that the gated recurrence's kernels share.
//
// Per feature and step, with r, i the gates' pre-activations and sig the sigmoid,
//     u = |alpha| sig(r),   a = exp(-u),   w = 1 - a,
//     m = sqrt(1 - a^2) = sqrt(w (2 - w)),   b = m sig(i) x,
//     h = a h_before + b   (h = b at a begin step).
// A slow decay (u up to 1/2) is carried as what it takes away, w, right to 2^-23 of
// itself, and applied as h_before - w h_before + b: a float a near 1 is off by up to
// 2^-25, at every step the same way where a gate stands still, and a memory of 1 / w
// steps with it by 2^-25 / w (3e-4 at w = 1e-4); m would lose the same digits to 1 - a^2.
// A fast one is a itself, off by u 2^-24 of it (the exponent's product): what little it
// leaves of a state has to be right, too.  (An infinite state turns into NaN under a slow
// decay: inf - inf.)
#pragma once

#include "scan_common.hpp"
#include "kernels.hpp"

namespace memoroid {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLog2eLow = 1.92596299112661746e-08f;    // log2(e) less the float above
constexpr float kSlow = 0.5f;                            // decays up to exp(-1/2) are slow

// exp(-v).  FAST, for bf16 gates, whose own steps are 2^-9 of v and move the result by far
// more: one rounded product into the hardware's 2^y, off by |v| 2^-24; else
// by 2^-23 whatever v (the product's integer part taken out before it can cost the
// fraction its digits).  v = NaN stays, +-inf give 0 and inf.
template <bool FAST>
__device__ __forceinline__ float exp_minus(float v) {
    if constexpr (FAST) return __builtin_amdgcn_exp2f(v * -kLog2e);
    // (past 2^+-300 everything is 0 or inf, and n below stays far from overflow)
    v = v > 300.0f ? 300.0f : v < -300.0f ? -300.0f : v;
    const float n = __builtin_rintf(v * -kLog2e);
    float f = __builtin_fmaf(v, -kLog2e, -n);
    f = __builtin_fmaf(v, -kLog2eLow, f);
    return __builtin_ldexpf(__builtin_amdgcn_exp2f(f), (int)n);
}
template <bool FAST>
__device__ __forceinline__ float sigmoid(float v) {
    return __builtin_amdgcn_rcpf(1.0f + exp_minus<FAST>(v));
}

// 1 - exp(-u) for 0 <= u <= 1/2: minimax fits of (1 - exp(-u)) / u there with the
// constant 1.  Relative error with the roundings 2^-23; FAST: 2^-22.
template <bool FAST>
__device__ __forceinline__ float loss_of(float u) {
    float p;
    if constexpr (FAST) {
        p = 0x1.bf3082p-8f;
        p = __builtin_fmaf(p, u, -0x1.5058b2p-5f);
        p = __builtin_fmaf(p, u, 0x1.5521aap-3f);
        p = __builtin_fmaf(p, u, -0x1.fffebp-2f);
    } else {
        p = -0x1.27c254p-10f;
        p = __builtin_fmaf(p, u, 0x1.0c9214p-7f);
        p = __builtin_fmaf(p, u, -0x1.550f3ep-5f);
        p = __builtin_fmaf(p, u, 0x1.555374p-3f);
        p = __builtin_fmaf(p, u, -0x1.fffff8p-2f);
    }
    return __builtin_fmaf(p, u, 1.0f) * u;
}

// A decay by exp(-u), u >= 0, in one float k: a slow one is minus what it takes away
// (its sign bit set, for u = 0 too), a fast one what it leaves.  SLOW: the caller knows
// that no u is above kSlow.
template <bool SLOW, bool FAST = false>
struct Decay {
    float k;
    __device__ __forceinline__ Decay() {}
    __device__ __forceinline__ explicit Decay(float u) {
        k = -loss_of<FAST>(u);
        if constexpr (!SLOW) {
            const float a = __builtin_amdgcn_exp2f(u * -kLog2e);
            k = u <= kSlow ? k : a;
        }
    }
    __device__ __forceinline__ bool slow() const { return SLOW || (int)__float_as_uint(k) < 0; }
    __device__ __forceinline__ float left() const { return slow() ? 1.0f + k : k; }          // a
    __device__ __forceinline__ float taken() const { return slow() ? -k : 1.0f - k; }        // w
    // a v + add
    __device__ __forceinline__ float of(float v, float add) const {
        const float t = __builtin_fmaf(k, v, add);
        return slow() ? v + t : t;
    }
    __device__ __forceinline__ float of(float v) const {
        const float t = k * v;
        return SLOW ? __builtin_fmaf(k, v, v) : slow() ? __builtin_fmaf(k, v, v) : t;
    }
};

// A feature's gates at one step
template <bool FAST, bool SLOW>
struct Gate {
    float sr, si, u, m;
    Decay<SLOW, FAST> decay;
    __device__ __forceinline__ Gate(float r, float i, float rate)
        : sr(sigmoid<FAST>(r)), si(sigmoid<FAST>(i)), u(rate * sr), decay(u) {
        const float w = decay.taken();
        m = __builtin_amdgcn_sqrtf(w * (2.0f - w));
    }
};

// ------------------------------------------------------------------ tiles
// A workgroup has kGateCols features of a tape (a chain) and kRuns runs of L steps, one
// behind the other.  A lane has F features of a run, so kRow of them a run's all.  (F = 2:
// 64 features of bf16 are one 128-byte line; with four a lane registers halve the steps.)
template <int F, int THREADS>
struct Lanes {
    static constexpr int kRow = kGateCols / F, kRuns = THREADS / kRow;
    static_assert(kRow <= 64 && kRuns <= 32, "a run lies in a wavefront, the runs' flags in a word");
};

// Rows of a tile in memory: the resource with the range check, and the bare address
struct Rows {
    Rsrc r;
    char* p;
};
__device__ __forceinline__ Rows rows_at(const void* p, int64_t bytes) { return {make_rsrc(p, bytes), (char*)p}; }

// 4 bytes at an address that is a multiple of 2
typedef uint32_t Word2 __attribute__((aligned(2)));

// Two features as they lie in memory.  FULL: rows and addresses are multiples of two
// elements, accesses go through the resource.  Otherwise rows start at any element: in bf16
// one access at that alignment, which the hardware takes; the last feature of an odd row comes
// with the one before it and is moved down by settle(), when nobody waits for it any more.
template <bool BF16>
struct Few {
    static constexpr int SIZE = BF16 ? 2 : 4, WORDS = BF16 ? 1 : 2;
    uint32_t w[WORDS];
    // off, soff: bytes from the tile's first row, a lane's and a scalar part, the latter not
    // covered by the range check; in: the row is one of the tape's; wide: rows of more than one
    template <int AUX, bool FULL>
    __device__ __forceinline__ void load(const Rows& m, uint32_t off, uint32_t soff, int left, bool in, bool wide) {
        if constexpr (FULL && BF16) {
            w[0] = __builtin_amdgcn_raw_buffer_load_b32(m.r, (int)off, (int)soff, AUX);
        } else if constexpr (FULL) {
            const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(m.r, (int)off, (int)soff, AUX);
            w[0] = v.x;
            w[1] = v.y;
        } else {
#pragma unroll
            for (int e = 0; e < WORDS; ++e) w[e] = 0u;
            if (!in || left <= 0) return;
            const char* const at = m.p + soff;
            if constexpr (BF16) {
                if (wide) w[0] = *(const Word2*)(at + (off - (left == 1 ? SIZE : 0)));
                else w[0] = *(const uint16_t*)(at + off);
            } else {
                // (8 bytes in one access at a multiple of 4 are slower: 156 -> 183 us, 8 x 4096 x 1023)
                w[0] = *(const uint32_t*)(at + off);
                if (left > 1) w[1] = *(const uint32_t*)(at + (off + SIZE));
            }
        }
    }
    template <bool FULL>
    __device__ __forceinline__ void settle(int left, bool wide) {
        if constexpr (!FULL && BF16) w[0] = left == 1 && wide ? w[0] >> 16 : w[0];
    }
    template <int AUX, bool FULL>
    __device__ __forceinline__ void store(const Rows& m, uint32_t off, uint32_t soff, int left, bool in) const {
        if constexpr (FULL && BF16) {
            __builtin_amdgcn_raw_buffer_store_b32(w[0], m.r, (int)off, (int)soff, AUX);
        } else if constexpr (FULL) {
            const u32x2 v = {w[0], w[1]};
            __builtin_amdgcn_raw_buffer_store_b64(v, m.r, (int)off, (int)soff, AUX);
        } else {
            if (!in || left <= 0) return;
            char* const at = m.p + soff;
            if (left == 1) {
                if constexpr (BF16) *(uint16_t*)(at + off) = (uint16_t)w[0];
                else *(uint32_t*)(at + off) = w[0];
            } else {
                if constexpr (BF16) *(Word2*)(at + off) = w[0];
                else {
                    *(uint32_t*)(at + off) = w[0];
                    *(uint32_t*)(at + (off + SIZE)) = w[1];
                }
            }
        }
    }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (BF16) return e & 1 ? bf16_hi(w[e / 2]) : bf16_lo(w[e / 2]);
        else return __uint_as_float(w[e]);
    }
    __device__ __forceinline__ void set(const float (&v)[2]) {
#pragma unroll
        for (int e = 0; e < WORDS; ++e) w[e] = BF16 ? f32x2_to_bf16x2(v[2 * e], v[2 * e + 1]) : __float_as_uint(v[e]);
    }
    // hides that what follows could be formed from what came before
    __device__ __forceinline__ void opaque() {
#pragma unroll
        for (int e = 0; e < WORDS; ++e) asm volatile("" : "+v"(w[e]));
    }
};

// The chain of a workgroup and its tile there: the n-th to start, so that all tiles
// before it are running or done; one thread asks, `shared` hands it on.
struct TileOf {
    int64_t tile;
    int chain;
};
__device__ __forceinline__ TileOf take_tile(const GatedTiles& t, uint32_t* shared) {
    // Every chain once per nchains workgroups.  Neighbouring chains run side by side on one
    // accelerator die (workgroup g on die g mod kXcds), whose cache then serves the lines that
    // both have a part of, and no chain stays on one die.
    const uint32_t nch = (uint32_t)t.nchains, i = blockIdx.x % nch, turn = blockIdx.x / nch, each = nch / kXcds, rest = nch % kXcds;
    const uint32_t die = rest ? i % kXcds : (i + turn) % kXcds;
    TileOf r;
    r.chain = (int)(die * each + (die < rest ? die : rest) + i / kXcds);
    r.tile = 0;
    if (t.nt > 1) {
        if (threadIdx.x == 0)
            *shared = claim_of(take_ticket(t.ctr + (size_t)r.chain * kCtrStride, (uint32_t)t.nt), (uint32_t)t.nt).pos;
        barrier_lds();
        r.tile = (int64_t)__builtin_amdgcn_readfirstlane(*shared);
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (t.nt == 1) t.hdr->timeout = kEmpty32;          // (else the fill before this kernel has written it)
        t.hdr->sig = t.sig;
    }
    return r;
}

// Words that tiles hand on, per feature: AGG, a tile without a begin step, as its decay
// and what it adds; INCL, the value after the tile.  Unpublished: all ones.
__device__ __forceinline__ void put_agg(const GatedTiles& t, int64_t slot, int f, float k, float add) {
    publish64(t.agg + slot * kGateCols + f, pack2(k, add));
}
__device__ __forceinline__ void put_incl(const GatedTiles& t, int64_t slot, int f, float v) {
    publish32(t.incl + slot * kGateCols + f, __float_as_uint(canon(v)));
}

// The value that enters a tile, a lane per feature: that of the nearest tile before it
// that has published its own, the ones between applied one after the other.  Each of them
// does the same for its own, so the result is the same bit for bit whichever tile that
// was.  First one wavefront tries: the word of the tile right before (which mostly is
// there where chains are many), then once the four nearest tiles.  If that is not
// enough, all wavefronts look at kNear tiles at a time, and the first puts what they
// found together: where chains are few and long, that is what sets the pace (one chain of
// 1024 tiles, fp32, no episode's begin: 99 us, 28 without the look-back).  48 tiles take 101 there,
// 64 93, but their LDS costs others more (8 x 4096 x 2048 bf16 117 -> 132 and 135 us).
constexpr int kNear = 32;
constexpr float kIsValue = 2.0f, kIsEmpty = 3.0f;                    // in the place of a decay's k, which is below 1
struct LookBackLds {
    float k[kNear][kGateCols], v[kNear][kGateCols];
    uint32_t done;
};

__device__ __forceinline__ bool try_near(const GatedTiles& t, int64_t tile, int chain, int f, bool need, float& v) {
    constexpr int W = 4;
    // (the words' addresses: scalars, and the lane's 32 bits)
    const int64_t stride = (int64_t)t.nchains * kGateCols, from = ((tile - 1) * t.nchains + chain) * kGateCols;
    v = 0.0f;
    bool done = !need;
    if (need) {
        const uint32_t w = peek32(t.incl + from + f);
        v = __uint_as_float(w);
        done = w != kEmpty32;
    }
    for (uint32_t polls = 0; !__all(done); ++polls) {
        if (polls == t.near) return false;
        if (polls) __builtin_amdgcn_s_sleep(1);
        uint32_t in[W];
        uint64_t ag[W];
#pragma unroll
        for (int k = 0; k < W; ++k) {
            in[k] = kEmpty32;
            ag[k] = kEmpty64;
            if (k < tile) {
                in[k] = peek32(t.incl + (from - k * stride) + f);
                ag[k] = peek64(t.agg + (from - k * stride) + f);
            }
        }
        int at = W;
#pragma unroll
        for (int k = W - 1; k >= 0; --k) at = in[k] != kEmpty32 ? k : at;
        bool ready = at < W && !done;
#pragma unroll
        for (int k = 0; k < W - 1; ++k) ready = ready && (k >= at || ag[k] != kEmpty64);
#pragma unroll
        for (int k = W - 1; k >= 0; --k) {
            Decay<false> d;
            d.k = unpack_lo(ag[k]);
            const float next = d.of(v, unpack_hi(ag[k]));
            v = !ready || k > at ? v : k == at ? __uint_as_float(in[k]) : next;
        }
        done = done || ready;
    }
    return true;
}

// All wavefronts of the workgroup; `use` is called by the first with the value.  WORDS: of a
// batch whose latencies are one, as many as a tile's registers leave room for
template <int THREADS, int WORDS, class Use>
__device__ __forceinline__ void look_far(const GatedTiles& t, int64_t tile, int chain, int f, bool need, LookBackLds& lds,
                                         Use use) {
    constexpr int kEach = kNear / (THREADS / 64);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t stride = (int64_t)t.nchains * kGateCols, from = ((tile - 1) * t.nchains + chain) * kGateCols;
    for (uint32_t polls = 0;; ++polls) {
#pragma unroll
        for (int n0 = 0; n0 < kEach; n0 += WORDS) {
            uint32_t in[WORDS];
            uint64_t ag[WORDS];
#pragma unroll
            for (int k = 0; k < WORDS; ++k) {
                const int n = wave * kEach + n0 + k;
                in[k] = kEmpty32;
                ag[k] = kEmpty64;
                if (n < tile && need) {
                    in[k] = peek32(t.incl + (from - n * stride) + f);
                    ag[k] = peek64(t.agg + (from - n * stride) + f);
                }
            }
#pragma unroll
            for (int k = 0; k < WORDS; ++k) {
                const int n = wave * kEach + n0 + k;
                const bool is = in[k] != kEmpty32;
                lds.k[n][lane] = is ? kIsValue : ag[k] != kEmpty64 ? unpack_lo(ag[k]) : kIsEmpty;
                lds.v[n][lane] = is ? __uint_as_float(in[k]) : unpack_hi(ag[k]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        barrier_lds();
        if (wave == 0) {
            // (a block at a time: read one by one they cost LDS's latency each)
            constexpr int kBlock = WORDS;
            int at = kNear;                                          // the nearest value
            bool ready = !need;
            for (int n0 = 0; n0 < kNear && !__all(ready || at < kNear); n0 += kBlock) {
                float k[kBlock];
#pragma unroll
                for (int j = 0; j < kBlock; ++j) k[j] = lds.k[n0 + j][lane];
#pragma unroll
                for (int j = 0; j < kBlock; ++j) {
                    if (at == kNear && k[j] == kIsValue) at = n0 + j;
                    if (at == kNear && k[j] == kIsEmpty) at = kNear + 1;    // not there yet
                }
            }
            ready = ready || at < kNear;
            const bool all = __all(ready);
            const bool late = polls >= kMaxPolls;
            if (all || late) {
                const bool found = need && at < kNear;
                float v = found ? lds.v[at][lane] : 0.0f;
                for (int n0 = kNear - kBlock; n0 >= 0; n0 -= kBlock) {
                    if (!__any(found && n0 < at)) continue;
                    float k[kBlock], add[kBlock];
#pragma unroll
                    for (int j = 0; j < kBlock; ++j) {
                        k[j] = lds.k[n0 + j][lane];
                        add[j] = lds.v[n0 + j][lane];
                    }
#pragma unroll
                    for (int j = kBlock - 1; j >= 0; --j) {
                        Decay<false> d;
                        d.k = k[j];
                        const float next = d.of(v, add[j]);
                        v = found && n0 + j < at ? next : v;
                    }
                }
                if (!all) flag_timeout(&t.hdr->timeout);
                use(v);
            } else {
                __builtin_amdgcn_s_sleep(1);
            }
            if (lane == 0) lds.done = all || late;
        }
        barrier_lds();
        if (lds.done) return;
    }
}

}  // namespace memoroid
