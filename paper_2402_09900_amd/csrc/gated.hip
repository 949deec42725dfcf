// gated.hip -- the gated linear recurrence over tapes of episodes, its gradient and
// its single step.  Formulas and their arithmetic: gated_common.hpp.
//
// Gradient, with g = dL/dh, lam = dL/dh with what later steps add,
//     lam_t = g_t + c_t,   c_{t-1} = a_t lam_t  (0 at a begin step),
//     dx = lam m sig(i),   di = lam b (1 - sig(i)),
//     du = lam (sig(i) x a^2 / m - a h_before),   dr = du u (1 - sig(r)),
//     dalpha = sign(alpha) sum du sig(r).
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
__global__ __launch_bounds__(64) void gated_bwd_kernel(GatedBwdArgs p) {
    __shared__ float before[kGateStateSteps][64];
    const int64_t nfb = (p.d + 63) / 64, b = blockIdx.x / nfb, f = (blockIdx.x - b * nfb) * 64 + threadIdx.x;
    if (f >= p.d) return;
    const float rate = __builtin_fabsf(p.alpha[f]);
    const int64_t ns = (p.T + kGateStateSteps - 1) / kGateStateSteps;
    float c = p.grad_state ? p.grad_state[b * p.d + f] : 0.0f;
    double sum = 0.0;
    for (int64_t s = ns - 1; s >= 0; --s) {
        const int64_t t0 = s * kGateStateSteps;
        const int n0 = (int)(p.T - t0 < kGateStateSteps ? p.T - t0 : kGateStateSteps);
        float h = p.states[(b * ns + s) * p.d + f];
        for (int k = 0; k < n0; ++k) {
            const int64_t n = b * p.T + t0 + k;
            const Gate<BF16, false> g(value<BF16>(p.gates, 2 * n * p.d + f),
                                                value<BF16>(p.gates, (2 * n + 1) * p.d + f), rate);
            const float v = g.m * g.si * value<BF16>(p.x, n * p.d + f);
            const bool begin = p.start[n] != 0;
            before[k][threadIdx.x] = begin ? 0.0f : h;
            h = begin ? v : g.decay.of(h, v);
        }
        for (int k = n0 - 1; k >= 0; --k) {
            const int64_t n = b * p.T + t0 + k;
            const float x = value<BF16>(p.x, n * p.d + f);
            const Gate<BF16, false> g(value<BF16>(p.gates, 2 * n * p.d + f),
                                                value<BF16>(p.gates, (2 * n + 1) * p.d + f), rate);
            const float a = g.decay.left();
            const float lam = value<BF16>(p.g, n * p.d + f) + c;
            const float rm = g.m > 0.0f ? 1.0f / g.m : 0.0f;
            const float du = lam * a * (g.si * x * a * rm - before[k][threadIdx.x]);
            put<BF16>(p.dx, n * p.d + f, lam * g.m * g.si);
            put<BF16>(p.dgates, 2 * n * p.d + f, du * rate * g.sr * (1.0f - g.sr));
            put<BF16>(p.dgates, (2 * n + 1) * p.d + f, lam * g.m * g.si * x * (1.0f - g.si));
            sum += (double)(du * g.sr);
            c = p.start[n] ? 0.0f : g.decay.of(lam, 0.0f);
        }
    }
    if (p.grad_state_in) p.grad_state_in[b * p.d + f] = c;
    if (p.part) p.part[b * p.d + f] = (float)sum;
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

hipError_t gated_bwd_launch(bool bf16, const GatedBwdArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)((a.d + 63) / 64 * a.B));
    if (bf16) hipLaunchKernelGGL(gated_bwd_kernel<true>, grid, dim3(64), 0, s, a);
    else hipLaunchKernelGGL(gated_bwd_kernel<false>, grid, dim3(64), 0, s, a);
    if (!a.part) return hipGetLastError();
    hipLaunchKernelGGL(gated_alpha_kernel, dim3((unsigned)((a.d + 63) / 64)), dim3(1024), 0, s, a.part, a.alpha, a.dalpha, a.part_rows, a.d);
    return hipGetLastError();
}

hipError_t gated_step_launch(bool bf16, const GatedStepArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)((a.B * a.d + 255) / 256));
    if (bf16) hipLaunchKernelGGL(gated_step_kernel<true>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(gated_step_kernel<false>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace memoroid
