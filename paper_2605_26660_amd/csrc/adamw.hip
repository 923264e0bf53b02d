// windq_adamw: one AdamW step over many tensors at once, moments in 32 bits or in 8.
//   m <- b1 m + (1 - b1) g     v <- b2 v + (1 - b2) g^2     p <- p decay - size m / (sqrt(v) inverse + eps)
// Every value is read once and written once and nothing else moves: 28 bytes a parameter with fp32 moments, 16 with 8-bit
// ones, against some 75 vector instructions in 8 bits, so HBM is what bounds it but for bfloat16 parameters.
//   A launch takes up to AW_MANY tensors: their descriptors travel in the kernel arguments and a workgroup finds its tensor by
// bisection over first-tile numbers.  A workgroup has AW_TILE consecutive values; a wavefront reads 256 of them at a time,
// four a lane, so that the block that shares an 8-bit scale is exactly a wavefront's step: its largest magnitude is a butterfly
// over 64 lanes and no value is visited twice.
//   Magnitudes are compared as integers (a float's bits without its sign): NaN and infinities order above all else and cannot
// get lost in a maximum.
//   45 M parameters, fp32 moments, bfloat16 gradients and copy 249 us (5.1 TB/s); 448 tensors of 65536 in 8 bits 110 us in two launches of 46 to 49 us (4.9 TB/s
// in each).  In 8 bits with bfloat16 parameters (8 bytes a parameter) the instructions take as long as the bytes: 6.5 M in 37 ragged tensors 22.5 us, 21.3 in
// one tensor (12.7 us of instruction issue, 12.5 us of bytes, in one generation of workgroups that load, compute and store about in step).
#include <math.h>
#include <string.h>

#include "windq_common.hpp"

namespace windq {

constexpr int AW_THREADS = 256;
constexpr int AW_STEPS = 4;                               // blocks of 256 values a wavefront takes
constexpr int64_t AW_TILE = (int64_t)AW_THREADS * 4 * AW_STEPS;
// Tensors of a launch.  AW_MANY is what keeps the arguments below 16 KB; 448 tensors of 65536 in 8 bits, one after the other on the same data: 224 a launch 95 us,
// 112 a launch 115, 64 a launch 137.  Up to AW_FEW they take 1 KB of arguments: two tensors of 8192 5.7 us and 6.3, sixteen 5.9 and 6.4.
constexpr int AW_FEW = 16, AW_MANY = 224;

struct AdamwRates {
    float b1, c1, b2, c2, eps, decay, size, inverse;
};

template <int N>
struct AdamwBatch {
    int32_t n;
    AdamwRates r;
    const float* grad_scale;
    uint32_t tile_start[N];
    windq_adamw_item t[N];
};

typedef float f32x2 __attribute__((ext_vector_type(2)));

template <typename T>
__device__ __forceinline__ void aw_load4(const T* __restrict__ p, int64_t i, int64_t n, bool whole, float (&x)[4]) {
    if (whole) {
        if constexpr (sizeof(T) == 4) {
            const float4 q = *reinterpret_cast<const float4*>(p + i);
            x[0] = q.x; x[1] = q.y; x[2] = q.z; x[3] = q.w;
        } else {
            const uint2 q = *reinterpret_cast<const uint2*>(p + i);
            x[0] = bf16_bits_to_f32(q.x & 0xffffu); x[1] = __uint_as_float(q.x & 0xffff0000u);
            x[2] = bf16_bits_to_f32(q.y & 0xffffu); x[3] = __uint_as_float(q.y & 0xffff0000u);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[j] = 0.0f;
        if (i + j < n) {
            if constexpr (sizeof(T) == 4) x[j] = p[i + j];
            else x[j] = bf16_bits_to_f32(p[i + j]);
        }
    }
}

__device__ __forceinline__ uint16_t aw_bf16(float x) {
    const __bf16 b = (__bf16)x;                            // one instruction: to nearest, ties to even, NaN kept
    return __builtin_bit_cast(uint16_t, b);
}

template <typename T>
__device__ __forceinline__ void aw_store4(T* __restrict__ p, int64_t i, int64_t n, bool whole, const float (&x)[4]) {
    if (whole) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(p + i) = make_float4(x[0], x[1], x[2], x[3]);
        } else {
            *reinterpret_cast<uint2*>(p + i) = make_uint2(aw_bf16(x[0]) | (uint32_t)aw_bf16(x[1]) << 16, aw_bf16(x[2]) | (uint32_t)aw_bf16(x[3]) << 16);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (i + j < n) {
            if constexpr (sizeof(T) == 4) p[i + j] = x[j];
            else p[i + j] = aw_bf16(x[j]);
        }
    }
}

// Four 8-bit values as one word; past the tensor's end zeros.
__device__ __forceinline__ uint32_t aw_load_word(const uint8_t* __restrict__ p, int64_t i, int64_t n, bool whole) {
    if (whole) return *reinterpret_cast<const uint32_t*>(p + i);
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < n) w |= (uint32_t)p[i + j] << (8 * j);
    return w;
}

__device__ __forceinline__ void aw_store_word(uint8_t* __restrict__ p, int64_t i, int64_t n, bool whole, uint32_t w) {
    if (whole) {
        *reinterpret_cast<uint32_t*>(p + i) = w;
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < n) p[i + j] = (uint8_t)(w >> (8 * j));
}

__device__ __forceinline__ void aw_decode(uint32_t w, float scale, float (&x)[4]) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo.x * scale; x[1] = lo.y * scale; x[2] = hi.x * scale; x[3] = hi.y * scale;
}

__device__ __forceinline__ uint32_t aw_encode(const float (&t)[4]) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], w, true);
}

__device__ __forceinline__ uint32_t aw_magnitude(const float (&x)[4]) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) m = max(m, __float_as_uint(x[j]) & 0x7fffffffu);
    return m;
}

// A block's scale from its largest magnitude, and the factor that brings its values to the type's range.
__device__ __forceinline__ float aw_scale(uint32_t largest, float& inverse) {
    const float scale = __uint_as_float(largest) * (float)(1.0 / 448.0);
    const bool whole = scale >= 1.17549435e-38f;
    inverse = whole ? 1.0f / scale : 0.0f;
    return whole ? scale : 0.0f;
}

template <typename P, typename GR, int BITS, int N>
__global__ __launch_bounds__(AW_THREADS) void adamw_kernel(const AdamwBatch<N> B) {
    int lo = 0, hi = B.n;                                  // the last tensor whose first tile is not past this one
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (B.tile_start[mid] <= blockIdx.x) lo = mid;
        else hi = mid;
    }
    const windq_adamw_item& T = B.t[lo];
    const int64_t n = T.n;
    const AdamwRates R = B.r;
    const float gs = B.grad_scale != nullptr ? *B.grad_scale : 1.0f;
    P* __restrict__ const p = static_cast<P*>(T.p);
    const GR* __restrict__ const g = static_cast<const GR*>(T.g);
    uint16_t* __restrict__ const copy = static_cast<uint16_t*>(T.copy);
    const uintptr_t at = reinterpret_cast<uintptr_t>(T.m) | reinterpret_cast<uintptr_t>(T.v);
    const bool even = (reinterpret_cast<uintptr_t>(p) & (4 * sizeof(P) - 1)) == 0 && (reinterpret_cast<uintptr_t>(g) & (4 * sizeof(GR) - 1)) == 0 &&
                      (at & (BITS == 8 ? 3 : 15)) == 0 && (reinterpret_cast<uintptr_t>(copy) & 7) == 0;
    const int64_t base = (int64_t)(blockIdx.x - B.tile_start[lo]) * AW_TILE + (threadIdx.x >> 6) * 256 + (threadIdx.x & 63) * 4;

    float pv[AW_STEPS][4], gv[AW_STEPS][4], mv[AW_STEPS][4], vv[AW_STEPS][4];
    uint32_t mw[AW_STEPS], vw[AW_STEPS];
    float ms[AW_STEPS], vs[AW_STEPS];
#pragma unroll
    for (int s = 0; s < AW_STEPS; ++s) {
        const int64_t i = base + s * (AW_THREADS * 4);
        const bool whole = even && i + 4 <= n;
        aw_load4(g, i, n, whole, gv[s]);
        aw_load4(p, i, n, whole, pv[s]);
        if constexpr (BITS == 8) {
            mw[s] = aw_load_word(static_cast<const uint8_t*>(T.m), i, n, whole);
            vw[s] = aw_load_word(static_cast<const uint8_t*>(T.v), i, n, whole);
            ms[s] = i < n ? T.m_scale[i >> 8] : 0.0f;
            vs[s] = i < n ? T.v_scale[i >> 8] : 0.0f;
        } else {
            aw_load4(static_cast<const float*>(T.m), i, n, whole, mv[s]);
            aw_load4(static_cast<const float*>(T.v), i, n, whole, vv[s]);
        }
    }
#pragma unroll
    for (int s = 0; s < AW_STEPS; ++s) {
        const int64_t i = base + s * (AW_THREADS * 4);
        if (__builtin_expect(i - (threadIdx.x & 63) * 4 >= n, 0)) break;          // the same for a wavefront
        const bool whole = even && i + 4 <= n;
        if constexpr (BITS == 8) {
            aw_decode(mw[s], ms[s], mv[s]);
            aw_decode(vw[s], vs[s], vv[s]);
        }
        float root[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float gr = gv[s][j] * gs;
            const float old = BITS == 8 ? vv[s][j] * vv[s][j] : vv[s][j];
            mv[s][j] = mv[s][j] * R.b1 + gr * R.c1;
            vv[s][j] = old * R.b2 + (gr * gr) * R.c2;
            root[j] = sqrtf(vv[s][j]);
            pv[s][j] = pv[s][j] * R.decay - (mv[s][j] / (root[j] * R.inverse + R.eps)) * R.size;
        }
        aw_store4(p, i, n, whole, pv[s]);
        if (copy != nullptr) aw_store4(copy, i, n, whole, pv[s]);
        if constexpr (BITS == 8) {
            // lanes past the end hold zeros: p = m = g = 0 there, and v = 0
            uint32_t bm = aw_magnitude(mv[s]), br = aw_magnitude(root);
#pragma unroll
            for (int k = 32; k >= 1; k >>= 1) {
                bm = max(bm, (uint32_t)__shfl_xor((int)bm, k, 64));
                br = max(br, (uint32_t)__shfl_xor((int)br, k, 64));
            }
            float im, ir;
            const float sm = aw_scale(bm, im), sr = aw_scale(br, ir);
            float tm[4], tr[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                tm[j] = mv[s][j] * im;
                tr[j] = root[j] * ir;
                // what is nearer to 0 than to the smallest magnitude takes that one (sr = 0: the block is all zeros)
                if (root[j] > 0.0f && sr > 0.0f && tr[j] < 0.001953125f) tr[j] = 0.001953125f;
            }
            aw_store_word(static_cast<uint8_t*>(T.m), i, n, whole, aw_encode(tm));
            aw_store_word(static_cast<uint8_t*>(T.v), i, n, whole, aw_encode(tr));
            if ((threadIdx.x & 63) == 0) {
                T.m_scale[i >> 8] = sm;
                T.v_scale[i >> 8] = sr;
            }
        } else {
            aw_store4(static_cast<float*>(T.m), i, n, whole, mv[s]);
            aw_store4(static_cast<float*>(T.v), i, n, whole, vv[s]);
        }
    }
}

template <typename P, typename GR, int BITS, int N>
int adamw_launch(const windq_adamw_item* items, int count, const AdamwRates& r, const float* grad_scale, hipStream_t st) {
    AdamwBatch<N> B;
    B.n = count;
    B.r = r;
    B.grad_scale = grad_scale;
    int64_t tiles = 0;
    for (int k = 0; k < count; ++k) {
        B.tile_start[k] = (uint32_t)tiles;
        B.t[k] = items[k];
        tiles += (items[k].n + AW_TILE - 1) / AW_TILE;
    }
    adamw_kernel<P, GR, BITS, N><<<dim3((uint32_t)tiles), dim3(AW_THREADS), 0, st>>>(B);
    return hipGetLastError() == hipSuccess ? WINDQ_OK : WINDQ_EHIP;
}

template <typename P, typename GR, int BITS>
int adamw_all(const windq_adamw_item* items, int64_t n, const AdamwRates& r, const float* grad_scale, hipStream_t st) {
    windq_adamw_item some[AW_MANY];
    int count = 0;
    int64_t tiles = 0;
    for (int64_t k = 0; k <= n; ++k) {
        const int64_t more = k < n ? (items[k].n + AW_TILE - 1) / AW_TILE : 0;
        if (count > 0 && (k == n || count == AW_MANY || !fits_launch(tiles + more, AW_THREADS))) {
            const int status = count <= AW_FEW ? adamw_launch<P, GR, BITS, AW_FEW>(some, count, r, grad_scale, st)
                                               : adamw_launch<P, GR, BITS, AW_MANY>(some, count, r, grad_scale, st);
            if (status != WINDQ_OK) return status;
            count = 0;
            tiles = 0;
        }
        if (more > 0) {
            some[count++] = items[k];
            tiles += more;
        }
    }
    return WINDQ_OK;
}

}  // namespace windq

using namespace windq;

extern "C" int windq_adamw(const windq_adamw_item* items, int64_t n, int32_t p_dtype, int32_t g_dtype, int32_t state_bits,
                           int64_t step, double lr, double beta1, double beta2, double eps, double weight_decay,
                           const float* grad_scale, void* stream) {
    if (n < 0 || (n > 0 && items == nullptr)) return WINDQ_EINVAL;
    if ((p_dtype != WINDQ_F32 && p_dtype != WINDQ_BF16) || (g_dtype != WINDQ_F32 && g_dtype != WINDQ_BF16)) return WINDQ_EDTYPE;
    if (state_bits != 8 && state_bits != 32) return WINDQ_EINVAL;
    if (step < 1 || !(lr >= 0.0 && isfinite(lr)) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) ||
        !(eps > 0.0 && isfinite(eps)) || !(weight_decay >= 0.0 && isfinite(weight_decay)))
        return WINDQ_EINVAL;
    if (!((float)eps > 0.0f) || !aligned(grad_scale, 4)) return WINDQ_EINVAL;
    const size_t pb = p_dtype == WINDQ_F32 ? 4 : 2, gb = g_dtype == WINDQ_F32 ? 4 : 2, sb = state_bits == 32 ? 4 : 1;
    for (int64_t k = 0; k < n; ++k) {
        const windq_adamw_item& t = items[k];
        if (t.n < 0) return WINDQ_ESHAPE;
        if (t.n == 0) continue;
        if (t.p == nullptr || t.g == nullptr || t.m == nullptr || t.v == nullptr) return WINDQ_EINVAL;
        if (!aligned(t.p, pb) || !aligned(t.g, gb) || !aligned(t.m, sb) || !aligned(t.v, sb) || !aligned(t.copy, 2)) return WINDQ_EINVAL;
        if (state_bits == 8 && (t.m_scale == nullptr || t.v_scale == nullptr || !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))) return WINDQ_EINVAL;
        if (!fits_launch((t.n + AW_TILE - 1) / AW_TILE, AW_THREADS)) return WINDQ_ESHAPE;
    }
    AdamwRates r;
    r.b1 = (float)beta1;
    r.c1 = (float)(1.0 - beta1);
    r.b2 = (float)beta2;
    r.c2 = (float)(1.0 - beta2);
    r.eps = (float)eps;
    r.decay = (float)(1.0 - lr * weight_decay);
    r.size = (float)(lr / (1.0 - pow(beta1, (double)step)));
    r.inverse = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
    hipStream_t st = static_cast<hipStream_t>(stream);
#define WINDQ_AW(P, GR)                                                                        \
    (state_bits == 8 ? adamw_all<P, GR, 8>(items, n, r, grad_scale, st) : adamw_all<P, GR, 32>(items, n, r, grad_scale, st))
    if (p_dtype == WINDQ_F32) return g_dtype == WINDQ_F32 ? WINDQ_AW(float, float) : WINDQ_AW(float, uint16_t);
    return g_dtype == WINDQ_F32 ? WINDQ_AW(uint16_t, float) : WINDQ_AW(uint16_t, uint16_t);
#undef WINDQ_AW
}
