// What the kernels of a pair of packed matrices (windq_gated) share: the second matrix, the activation, and where the products go.
#pragma once

#include "windq_act.hpp"
#include "windq_adapters.hpp"

namespace windq {

struct PairArgs {
    PackArgs up;
    int32_t act;
    void* G;                   // [T][ld] the products, or both null
    void* U;
    int64_t ld_save;
};

#ifdef __HIPCC__

template <typename YT>
__device__ __forceinline__ void store_y(YT* __restrict__ p, float v) {
    if constexpr (sizeof(YT) == 4) *p = v;
    else *p = (uint16_t)f32_to_bf16_bits(v);
}

// act(g) u, with both kept where they are wanted.
template <typename YT>
__device__ __forceinline__ float pair_result(const PairArgs& Q, int64_t t, int64_t row, float g, float u) {
    if (Q.G != nullptr) {
        store_y(static_cast<YT*>(Q.G) + t * Q.ld_save + row, g);
        store_y(static_cast<YT*>(Q.U) + t * Q.ld_save + row, u);
    }
    float none;
    return activation<false>(Q.act, g, none) * u;
}

#endif  // __HIPCC__

}  // namespace windq
