// gated_step.hip -- one step of the gated recurrence, the state updated in place
// (formulas: gated_common.hpp).
#include "gated_common.hpp"

namespace memoroid {

namespace {

// V features a lane (V 4: d is a multiple of 4 and addresses are of 4 elements).  Bound by
// the launch where a state is small (16 rows of 256 in fp32: 2.4 us of kernel, 4.0 a call),
// then by memory (512 rows of 2048 in bf16: 17 MB in 4.9 us).
template <bool BF16, int V>
__global__ __launch_bounds__(256) void gated_step_kernel(GatedStepArgs p) {
    // (B d < 2^31)
    const uint32_t d = (uint32_t)p.d, i = (blockIdx.x * 256u + threadIdx.x) * V;
    if (i >= (uint32_t)p.B * d) return;
    const uint32_t b = i / d, f = i - b * d;
    float x[V], r[V], g[V], s[V], rate[V];
    auto load = [](const void* q, int64_t n, float (&v)[V]) {
        if constexpr (BF16 && V == 4) {
            const u32x2 w = *(const u32x2*)((const uint16_t*)q + n);
            v[0] = bf16_lo(w.x);
            v[1] = bf16_hi(w.x);
            v[2] = bf16_lo(w.y);
            v[3] = bf16_hi(w.y);
        } else if constexpr (BF16) {
            v[0] = bf16_lo(((const uint16_t*)q)[n]);
        } else if constexpr (V == 4) {
            *(u32x4*)v = *(const u32x4*)((const float*)q + n);
        } else {
            v[0] = ((const float*)q)[n];
        }
    };
    load(p.x, i, x);
    load(p.gates, (int64_t)2 * b * d + f, r);
    load(p.gates, ((int64_t)2 * b + 1) * d + f, g);
    const bool begins = p.start && p.start[b] != 0;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        s[e] = p.state[i + e];
        rate[e] = __builtin_fabsf(p.alpha[f + e]);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const Gate<BF16, false> gate(r[e], g[e], rate[e]);
        const float add = gate.m * gate.si * x[e], on = gate.decay.of(s[e], add);
        s[e] = begins ? add : on;
    }
#pragma unroll
    for (int e = 0; e < V; ++e) p.state[i + e] = s[e];
    if constexpr (BF16 && V == 4) *(u32x2*)((uint16_t*)p.h + i) = u32x2{f32x2_to_bf16x2(s[0], s[1]), f32x2_to_bf16x2(s[2], s[3])};
    else if constexpr (BF16) ((uint16_t*)p.h)[i] = (uint16_t)f32_to_bf16(s[0]);
    else if constexpr (V == 4) *(u32x4*)((float*)p.h + i) = *(const u32x4*)s;
    else ((float*)p.h)[i] = s[0];
}

template <bool BF16, int V>
void step(const GatedStepArgs& a, hipStream_t s) {
    hipLaunchKernelGGL((gated_step_kernel<BF16, V>), dim3((unsigned)((a.B * a.d / V + 255) / 256)), dim3(256), 0, s, a);
}

}  // namespace

hipError_t gated_step_launch(bool bf16, bool full, const GatedStepArgs& a, hipStream_t s) {
    if (bf16) full ? step<true, 4>(a, s) : step<true, 1>(a, s);
    else full ? step<false, 4>(a, s) : step<false, 1>(a, s);
    return hipGetLastError();
}

}  // namespace memoroid
