// retention_step.hip -- one step of retention for every row of a batch, the
// state updated in place: acting in environments, generating tokens.
//
//     S <- gamma S + k^T v   (k^T v at a begin),   out = scale q S
//
// Bound by the state, read once and written once (2 x 4 dk dv bytes a head; q, k,
// v and out are a hundredth of it): 256 rows of 16 heads of 128 in 106 us, 5.1 TB/s;
// 16 rows of 4 heads of 64 in 4.  A workgroup takes 32 columns
// of one head's state, a 128-byte line of each of its rows: eight lanes a row, 32
// rows at a time, so that a head of 128 x 128 has all its loads in flight at once,
// and a small batch still spreads over the chip (16 rows of 4 heads of 64: 128
// workgroups).  gamma has 48 bits (Carry): the same rounding of it at every step would
// add up over a rollout (16384 steps at a rate of 1/4096: 1.1e-4 of the state, 2.5e-7 so).
#include "retention_common.hpp"

namespace memoroid {

template <int NP>
__device__ __forceinline__ float elem(const void* p, int64_t i) {
    if constexpr (NP == 1) return __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16);
    else return ((const float*)p)[i];
}

template <int NP>
__global__ __launch_bounds__(256) void ret_step_kernel(RetStepArgs p, int vblocks) {
    __shared__ f32x4 sSum[4][8];
    const int64_t bh = blockIdx.x / (unsigned)vblocks;
    const int64_t b = bh / p.H, h = bh % p.H;
    const int64_t kh = b * p.Hk + h / (p.H / p.Hk);
    const int col = (int)(blockIdx.x % (unsigned)vblocks) * 32 + (threadIdx.x & 7) * 4, row0 = threadIdx.x >> 3;
    const bool in = col < p.dv;                            // dv is a multiple of 8
    float* const S = p.state + bh * p.dk * p.dv + col;
    f32x4 s[kRetMaxDim / 32];
#pragma unroll
    for (int i = 0; i < kRetMaxDim / 32; ++i) {
        const int row = row0 + 32 * i;
        s[i] = in && row < p.dk ? *(const f32x4*)(S + row * p.dv) : zero4();
    }
    const bool begin = p.start && p.start[b] != 0;
    const Carry gamma = carry_of(fabs((double)p.alpha[h]), 1.0);
    f32x4 v = zero4(), o = zero4();
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = in ? elem<NP>(p.v, kh * p.dv + col + e) : 0.0f;
#pragma unroll
    for (int i = 0; i < kRetMaxDim / 32; ++i) {
        const int row = row0 + 32 * i;
        if (in && row < p.dk) {
            const float k = elem<NP>(p.k, kh * p.dk + row), q = elem<NP>(p.q, bh * p.dk + row);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[i][e] = __builtin_fmaf(k, v[e], begin ? 0.0f : gamma(s[i][e]));
                o[e] = __builtin_fmaf(q, s[i][e], o[e]);
            }
            *(f32x4*)(S + row * p.dv) = s[i];
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        o[e] += lanes_xor(o[e], 8);
        o[e] += lanes_xor(o[e], 16);
        o[e] += lanes_xor(o[e], 32);
    }
    if ((threadIdx.x & 63) < 8) sSum[threadIdx.x >> 6][threadIdx.x & 7] = o;
    __syncthreads();
    if (threadIdx.x < 8 && in) {
        const int c = threadIdx.x;
        const f32x4 t = ((sSum[0][c] + sSum[1][c]) + (sSum[2][c] + sSum[3][c])) * p.scale;
        const int64_t at = bh * p.dv + col;
        if (NP == 1) *(u32x2*)((uint16_t*)p.out + at) = u32x2{f32x2_to_bf16x2(t[0], t[1]), f32x2_to_bf16x2(t[2], t[3])};
        else *(f32x4*)((float*)p.out + at) = t;
    }
}

hipError_t ret_step_launch(int planes, const RetStepArgs& a, hipStream_t s) {
    const int vblocks = (a.dv + 31) / 32;
    const dim3 grid((unsigned)(a.B * a.H * vblocks)), block(256);
    if (planes == 1) hipLaunchKernelGGL((ret_step_kernel<1>), grid, block, 0, s, a, vblocks);
    else hipLaunchKernelGGL((ret_step_kernel<3>), grid, block, 0, s, a, vblocks);
    return hipGetLastError();
}

}  // namespace memoroid
