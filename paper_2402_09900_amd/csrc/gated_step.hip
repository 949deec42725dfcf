// gated_step.hip -- one step of the gated recurrence, the state updated in place
// (formulas: gated_common.hpp).
#include "gated_common.hpp"

namespace memoroid {

namespace {

template <bool BF16>
__device__ __forceinline__ float value(const void* p, int64_t i) {
    if constexpr (BF16) return bf16_lo(((const uint16_t*)p)[i]);
    else return ((const float*)p)[i];
}
template <bool BF16>
__device__ __forceinline__ void put(void* p, int64_t i, float v) {
    if constexpr (BF16) ((uint16_t*)p)[i] = (uint16_t)f32_to_bf16(v);
    else ((float*)p)[i] = v;
}

template <bool BF16>
__global__ __launch_bounds__(256) void gated_step_kernel(GatedStepArgs p) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= p.B * p.d) return;
    const int64_t b = i / p.d, f = i - b * p.d;
    const Gate<BF16, false> g(value<BF16>(p.gates, 2 * b * p.d + f),
                                        value<BF16>(p.gates, (2 * b + 1) * p.d + f), __builtin_fabsf(p.alpha[f]));
    const float v = g.m * g.si * value<BF16>(p.x, i);
    const float s = p.state[i];
    const float h = p.start && p.start[b] ? v : g.decay.of(s, v);
    p.state[i] = h;
    put<BF16>(p.h, i, h);
}

}  // namespace

hipError_t gated_step_launch(bool bf16, const GatedStepArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)((a.B * a.d + 255) / 256));
    if (bf16) hipLaunchKernelGGL(gated_step_kernel<true>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(gated_step_kernel<false>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace memoroid
