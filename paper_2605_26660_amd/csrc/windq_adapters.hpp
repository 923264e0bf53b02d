// Low-rank adapters beside a packed product: kernels that the way there and the way back share.
#pragma once

#include "windq_project.hpp"

namespace windq {

// ------------------------------------------------------------------------------------------------ h = A x, token by token
// (On the way back: dh = alpha B^T dY, with B transposed in A's place.)  A workgroup takes 16 ranks of one token, a wavefront four of them; lanes walk the columns, eight at a time.
template <typename XT>
__device__ __forceinline__ void load8(const XT* __restrict__ p, float (&v)[8]) {
    if constexpr (sizeof(XT) == 4) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
        const uint4 r = *reinterpret_cast<const uint4*>(p);
        v[0] = bf16_bits_to_f32(r.x & 0xffffu); v[1] = __uint_as_float(r.x & 0xffff0000u);
        v[2] = bf16_bits_to_f32(r.y & 0xffffu); v[3] = __uint_as_float(r.y & 0xffff0000u);
        v[4] = bf16_bits_to_f32(r.z & 0xffffu); v[5] = __uint_as_float(r.z & 0xffff0000u);
        v[6] = bf16_bits_to_f32(r.w & 0xffffu); v[7] = __uint_as_float(r.w & 0xffff0000u);
    }
}

template <typename XT>
__global__ __launch_bounds__(256) void shrink_token_kernel(const XT* __restrict__ X, int64_t ldx, int32_t cols, const AdapterArgs A,
                                                            bool scaled, float* __restrict__ h) {
    const int32_t groups = (A.max_rank + 15) >> 4;
    const int64_t t = blockIdx.x / groups;
    const int32_t r0 = (int32_t)(blockIdx.x - t * groups) * 16 + (threadIdx.x >> 6) * 4;
    if (r0 >= A.max_rank) return;                          // the same for a wavefront
    const int lane = threadIdx.x & 63;
    const int32_t k = A.of[t];
    const int32_t rank = k < 0 || k >= A.n ? 0 : adapter_rank(A, k);
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const float factor = scaled && rank > 0 && A.alpha != nullptr ? A.alpha[k] : 1.0f;
    if (r0 < rank) {
        const XT* __restrict__ const a = static_cast<const XT*>(A.a) + ((int64_t)k * A.max_rank + r0) * cols;
        const XT* __restrict__ const x = X + t * ldx;
#pragma unroll 2
        for (int32_t c = lane * 8; c < cols; c += 512) {
            float xv[8], av[8];
            load8(x + c, xv);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (r0 + i < rank) {
                    load8(a + (int64_t)i * cols + c, av);
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[i] = fmaf(av[j], xv[j], acc[i]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) acc[i] += __shfl_xor(acc[i], m, 64);
        if (lane == i && r0 + i < A.max_rank) h[t * A.max_rank + r0 + i] = factor * acc[i];
    }
}

}  // namespace windq
