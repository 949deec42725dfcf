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
// A fast one is a itself: what little it leaves of a state has to be right, too.
#pragma once

#include "scan_common.hpp"
#include "kernels.hpp"

namespace memoroid {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLog2eLow = 1.92596299112661746e-08f;    // log2(e) less the float above
constexpr float kSlow = 0.5f;                            // decays up to exp(-1/2) are slow

// exp(-v).  FAST: one rounded product into the hardware's 2^y, off by |v| 2^-24; else
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

// 1 - exp(-u) for 0 <= u <= 1/2, relative error 2^-23: a minimax fit of (1 - exp(-u)) / u
// there with the constant 1, relative error 2^-27.
__device__ __forceinline__ float loss_of(float u) {
    float p = -0x1.27c254p-10f;
    p = __builtin_fmaf(p, u, 0x1.0c9214p-7f);
    p = __builtin_fmaf(p, u, -0x1.550f3ep-5f);
    p = __builtin_fmaf(p, u, 0x1.555374p-3f);
    p = __builtin_fmaf(p, u, -0x1.fffff8p-2f);
    p = __builtin_fmaf(p, u, 1.0f);
    return p * u;
}

// A decay by exp(-u), u >= 0.  SLOW: the caller knows that no u is above kSlow.
template <bool SLOW>
struct Decay {
    float k;          // slow: minus what it takes away; else what it leaves
    bool slow;
    __device__ __forceinline__ explicit Decay(float u) {
        k = -loss_of(u);
        slow = true;
        if constexpr (!SLOW) {
            const float a = __builtin_amdgcn_exp2f(u * -kLog2e);
            slow = u <= kSlow;
            k = slow ? k : a;
        }
    }
    __device__ __forceinline__ float left() const { return slow ? 1.0f + k : k; }          // a
    __device__ __forceinline__ float taken() const { return slow ? -k : 1.0f - k; }        // w
    // a v + add
    __device__ __forceinline__ float of(float v, float add) const {
        const float t = __builtin_fmaf(k, v, add);
        return slow ? v + t : t;
    }
};

// A feature's gates at one step
template <bool FAST, bool SLOW>
struct Gate {
    float sr, si, u, m;
    Decay<SLOW> decay;
    __device__ __forceinline__ Gate(float r, float i, float rate)
        : sr(sigmoid<FAST>(r)), si(sigmoid<FAST>(i)), u(rate * sr), decay(u) {
        const float w = decay.taken();
        m = __builtin_amdgcn_sqrtf(w * (2.0f - w));
    }
};

}  // namespace memoroid
