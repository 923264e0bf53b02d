// dX of packed products on their way back: what windq_project_grad and windq_gated_grad share.
#pragma once

#include "windq_gemm.hpp"

namespace windq {

constexpr int DXF_TILES = 256;
constexpr size_t DXF_BYTES = (size_t)DXF_TILES * 64 * 64 * 4;      // of fp32's parts: tiles x splits are no more

struct DxArgs {
    PackArgs P;                // rows, cols alone where packed is false
    bool packed;
    const void* dY;            // rows on 16 bytes, readable up to a multiple of 8
    int64_t ldy;
    int64_t T;
    void* dX;
    int64_t ldx;
    const float* dh;           // [T][max_rank] or null
    AdapterArgs A;
    float* part;               // sums of parts of the rows; fp32: [splits][tiles][4][256][4], bfloat16: [splits][T][cols]
    int32_t splits;
    PackArgs up;               // of a pair: the second matrix and its side of the sum
    const void* dY_up;         // or null
};

int launch_dx_f32(DxArgs Q, hipStream_t st);

#ifdef __HIPCC__

__device__ __forceinline__ void skip_row(const PackArgs& P, int64_t row, int64_t col, float (&w)[8]) {
    if (P.w_f32 != 0) load8(static_cast<const float*>(P.W) + row * P.ld + col, w);
    else load8(static_cast<const uint16_t*>(P.W) + row * P.ld + col, w);
}

// An octet of one row as fp32 weights (rounded nowhere but by the multiply-add).
__device__ __forceinline__ void weight_octet(const PackArgs& P, int64_t row, int64_t col, const uint16_t* __restrict__ trits_of, float (&w)[8]) {
    const int64_t rb = row / P.R_u, lrow = row - rb * P.R_u;
    const int32_t j = (int32_t)(col / P.G), o = (int32_t)(col - (int64_t)j * P.G) >> 3;
    const int64_t u = rb * P.n_chunks + j;
    int64_t base;
    const int a = pk_action(P, u, base);
    if (a == 0) return skip_row(P, row, col, w);
    const int64_t g = u * P.R_u + lrow;
    const float s = P.scale[g], of = a >= 5 ? 0.0f : P.offset[g];
    const uint4 f = octet_fields(a, P.codes + base + lrow * pk_bytes_per_group(a, P.G), o, trits_of);
    const float f0 = pk_f0(a);
    const uint32_t m = P.mask != nullptr ? P.mask[row * P.mask_ld + (col >> 3)] : 0u;
    const uint32_t v[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = ((i & 1) != 0 ? __uint_as_float(v[i >> 1] & 0xffff0000u) : bf16_bits_to_f32(v[i >> 1] & 0xffffu)) - f0;
        w[i] = ((m >> i) & 1u) != 0u ? 0.0f : fmaf(q, s, of);
    }
}

// ROWS rows by eight columns of w_hat within a unit, whose treatment and first byte are known, put(row, column, weight) for each.
template <int ROWS, typename Put>
__device__ __forceinline__ void rows_of(const PackArgs& P, int64_t r0, int64_t col, int64_t u, int64_t lrow, int o, int a, int64_t base,
                                        const uint16_t* __restrict__ trits_of, Put put) {
    if (a == 0) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            float w[8];
            skip_row(P, r0 + i, col, w);
#pragma unroll
            for (int m = 0; m < 8; ++m) put(i, m, w[m]);
        }
        return;
    }
    const int32_t nb = (int32_t)pk_bytes_per_group(a, P.G);
    const uint8_t* const first = P.codes + base + lrow * nb;
    float sc[ROWS], of[ROWS];
    __builtin_memcpy(sc, P.scale + u * P.R_u + lrow, 4 * ROWS);
    __builtin_memcpy(of, P.offset + u * P.R_u + lrow, 4 * ROWS);
    uint4 f[ROWS];
    auto rows = [&](auto octet) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) f[i] = octet(first + i * nb);
    };
    switch (a) {
        case 1: rows([&](const uint8_t* p) { uint2 q; __builtin_memcpy(&q, p + o * 8, 8); return fields8(q.x, q.y); }); break;
        case 2: rows([&](const uint8_t* p) { uint32_t q; __builtin_memcpy(&q, p + o * 4, 4); return fields4(q); }); break;
        case 3: rows([&](const uint8_t* p) { return octet_fields(3, p, o, trits_of); }); break;
        case 4: rows([&](const uint8_t* p) { uint16_t q; __builtin_memcpy(&q, p + o * 2, 2); return fields2(q); }); break;
        case 5: rows([&](const uint8_t* p) { return fields2(octet_trits(p, o, trits_of) & 0xffffu); }); break;
        default: rows([&](const uint8_t* p) { return fields1(p[o]); }); break;
    }
    const float f0 = pk_f0(a);
    uint32_t m8[ROWS] = {};
    if (P.mask != nullptr) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) m8[i] = P.mask[(r0 + i) * P.mask_ld + (col >> 3)];
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
        for (int m = 0; m < 8; ++m) {
            const uint32_t pair = (m >> 1) == 0 ? f[i].x : ((m >> 1) == 1 ? f[i].y : ((m >> 1) == 2 ? f[i].z : f[i].w));
            const float q = ((m & 1) != 0 ? __uint_as_float(pair & 0xffff0000u) : __uint_as_float(pair << 16)) - f0;
            const float x = fmaf(q, sc[i], a >= 5 ? 0.0f : of[i]);
            put(i, m, ((m8[i] >> m) & 1u) != 0u ? 0.0f : x);
        }
}

// Eight rows by eight columns of w_hat; rows past the last one are zeros.
template <typename Put>
__device__ __forceinline__ void eight_rows(const PackArgs& P, int64_t r0, int64_t col, const uint16_t* __restrict__ trits_of, Put put) {
    const uint32_t R_u = (uint32_t)P.R_u, rb = (uint32_t)r0 / R_u, lrow = (uint32_t)r0 - rb * R_u;
    if (r0 + 8 <= P.rows && lrow + 8 <= R_u) {              // one unit's rows
        const uint32_t j = (uint32_t)col / (uint32_t)P.G;
        const int64_t u = (int64_t)rb * P.n_chunks + j;
        int64_t base;
        const int a = pk_action(P, u, base);
        rows_of<8>(P, r0, col, u, lrow, ((int)col - (int)j * P.G) >> 3, a, base, trits_of, put);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float w[8] = {};
            if (r0 + i < P.rows) weight_octet(P, r0 + i, col, trits_of, w);
#pragma unroll
            for (int m = 0; m < 8; ++m) put(i, m, w[m]);
        }
    }
}

// Fields as half precision numbers, two a word in their order: 4 + field, +-1, 16 + field, 8 + field as for bfloat16, three more bits of mantissa behind them.
__device__ __forceinline__ uint4 half_fields2(uint32_t v) {
    const uint32_t t = twice(v, 14, v);
    return make_uint4(((t << 8) & 0x03000300u) | 0x44004400u, ((t << 4) & 0x03000300u) | 0x44004400u, (t & 0x03000300u) | 0x44004400u, ((t >> 4) & 0x03000300u) | 0x44004400u);
}
__device__ __forceinline__ uint4 half_fields1(uint32_t v) {
    const uint32_t n = ~v, t = twice(n, 15, n & 0xffu);
    return make_uint4(((t << 15) & 0x80008000u) | 0x3c003c00u, ((t << 13) & 0x80008000u) | 0x3c003c00u, ((t << 11) & 0x80008000u) | 0x3c003c00u, ((t << 9) & 0x80008000u) | 0x3c003c00u);
}
__device__ __forceinline__ uint4 half_fields4(uint32_t v) {
    const uint32_t e = twice(v, 12, v & 0xffffu), o = twice(v >> 16, 12, v >> 16);
    return make_uint4(((e << 6) & 0x03c003c0u) | 0x4c004c00u, ((e >> 2) & 0x03c003c0u) | 0x4c004c00u, ((o << 6) & 0x03c003c0u) | 0x4c004c00u, ((o >> 2) & 0x03c003c0u) | 0x4c004c00u);
}
__device__ __forceinline__ uint4 half_fields3(uint32_t v) {
    return make_uint4(((v << 7) & 0x380u) | ((v << 20) & 0x3800000u) | 0x48004800u, ((v << 1) & 0x380u) | ((v << 14) & 0x3800000u) | 0x48004800u,
                      ((v >> 5) & 0x380u) | ((v << 8) & 0x3800000u) | 0x48004800u, ((v >> 11) & 0x380u) | ((v << 2) & 0x3800000u) | 0x48004800u);
}

// Two weights as half precision numbers: f scale + beta in fp32, rounded once.
__device__ __forceinline__ uint32_t half_pair(float lo, float hi) {
    return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)lo) | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)hi) << 16;
}

__device__ __forceinline__ uint4 half_fields8(uint32_t v0, uint32_t v1) {
    auto pair = [](uint32_t v, int lo) { return half_pair((float)((v >> (8 * lo)) & 0xffu), (float)((v >> (8 * lo + 8)) & 0xffu)); };
    return make_uint4(pair(v0, 0), pair(v0, 2), pair(v1, 0), pair(v1, 2));
}

__device__ __forceinline__ uint4 half_weights(uint4 f, float s, float b) {
    auto two = [&](uint32_t q) { return half_pair(fmaf((float)__builtin_bit_cast(_Float16, (uint16_t)q), s, b), fmaf((float)__builtin_bit_cast(_Float16, (uint16_t)(q >> 16)), s, b)); };
    return make_uint4(two(f.x), two(f.y), two(f.z), two(f.w));
}

// ROWS rows by eight columns of w_hat times `by`, a power of two, in half precision, within a unit whose treatment and first byte are known; no mask.  Five
// instructions a weight, where putting on the mask, the power and the centre one by one takes eleven.  Comes back with the columns that have something other than 0 (of codes: with none).
template <int ROWS>
__device__ __forceinline__ uint32_t half_rows(const PackArgs& P, int64_t r0, int64_t col, int64_t u, int64_t lrow, int o, int a, int64_t base, const uint16_t* __restrict__ trits_of,
                                              float by, uint4 (&w)[ROWS]) {
    if (a == 0) {
        uint4 all = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            float v[8];
            skip_row(P, r0 + i, col, v);
            w[i] = make_uint4(half_pair(v[0] * by, v[1] * by), half_pair(v[2] * by, v[3] * by), half_pair(v[4] * by, v[5] * by), half_pair(v[6] * by, v[7] * by));
            all = make_uint4(all.x | w[i].x, all.y | w[i].y, all.z | w[i].z, all.w | w[i].w);
        }
        const uint32_t pairs[4] = {all.x, all.y, all.z, all.w};
        uint32_t there = 0;
#pragma unroll
        for (int m = 0; m < 8; ++m) there |= (pairs[m >> 1] & ((m & 1) != 0 ? 0x7fff0000u : 0x7fffu)) != 0u ? 1u << m : 0u;
        return there;
    }
    const int32_t nb = (int32_t)pk_bytes_per_group(a, P.G);
    const uint8_t* const first = P.codes + base + lrow * nb;
    float sc[ROWS], be[ROWS];
    __builtin_memcpy(sc, P.scale + u * P.R_u + lrow, 4 * ROWS);
    __builtin_memcpy(be, P.offset + u * P.R_u + lrow, 4 * ROWS);
    uint4 f[ROWS];
    auto rows = [&](auto octet) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) f[i] = octet(first + i * nb);
    };
    switch (a) {
        case 1: rows([&](const uint8_t* p) {
            uint2 q;
            __builtin_memcpy(&q, p + o * 8, 8);
            return half_fields8(q.x, q.y);
        }); break;
        case 2: rows([&](const uint8_t* p) { uint32_t q; __builtin_memcpy(&q, p + o * 4, 4); return half_fields4(q); }); break;
        case 3: rows([&](const uint8_t* p) { return half_fields3((uint32_t)p[o * 3] | (uint32_t)p[o * 3 + 1] << 8 | (uint32_t)p[o * 3 + 2] << 16); }); break;
        case 4: rows([&](const uint8_t* p) { uint16_t q; __builtin_memcpy(&q, p + o * 2, 2); return half_fields2(q); }); break;
        case 5: rows([&](const uint8_t* p) { return half_fields2(octet_trits(p, o, trits_of) & 0xffffu); }); break;
        default: rows([&](const uint8_t* p) { return half_fields1(p[o]); }); break;
    }
    const float f0 = pk_f0(a);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const float s = sc[i] * by, b = fmaf(-f0, s, a >= 5 ? 0.0f : be[i] * by);
        w[i] = half_weights(f[i], s, b);
    }
    return 0;
}

template <typename HT>
__device__ __forceinline__ uint32_t half_bits(float x) {
    if constexpr (__is_same(HT, _Float16)) return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x);
    else return f32_to_bf16_bits(x);
}

// w_hat rounded to bfloat16 and turned: wt [cols][ld], zeros from the last row to K.  A thread has eight rows by eight columns.  In half precision (_Float16)
// weights are multiplied by a power of two first, the same for an octet of columns.  PLAIN: so, with no mask and whole eights of rows.  Comes back with a thread's columns that
// have something other than 0 (PLAIN: not of codes).
template <typename HT, bool PLAIN = false>
__device__ __forceinline__ uint32_t turn(const PackArgs& P, int32_t K, int64_t ld, float by, uint16_t* __restrict__ wt, int64_t block) {
    __shared__ uint16_t trits_of[256];
    trits_of[threadIdx.x] = (uint16_t)trit_fields(threadIdx.x);
    __syncthreads();
    const int32_t row_blocks = (K + 255) / 256;
    const int64_t cb = block / row_blocks;
    const int64_t r0 = (block - cb * row_blocks) * 256 + (threadIdx.x & 31) * 8, col = cb * 64 + (threadIdx.x >> 5) * 8;
    if (col >= P.cols || r0 >= K) return 0;
    uint32_t v[8][4], there = 0;
    if constexpr (PLAIN) {
        uint4 w[8] = {};
        if (r0 < P.rows) {
            const uint32_t R_u = (uint32_t)P.R_u, rb = (uint32_t)r0 / R_u, lrow = (uint32_t)r0 - rb * R_u;
            const uint32_t j = (uint32_t)col / (uint32_t)P.G;
            const int64_t u = (int64_t)rb * P.n_chunks + j;
            int64_t base;
            const int a = pk_action(P, u, base);
            there = half_rows<8>(P, r0, col, u, lrow, ((int)col - (int)j * P.G) >> 3, a, base, trits_of, by, w);
        }
#pragma unroll
        for (int m = 0; m < 8; ++m) {
            uint32_t t[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                auto word = [&](uint4 x) { return (m >> 1) == 0 ? x.x : ((m >> 1) == 1 ? x.y : ((m >> 1) == 2 ? x.z : x.w)); };
                t[i] = __builtin_amdgcn_perm(word(w[2 * i + 1]), word(w[2 * i]), (m & 1) != 0 ? 0x07060302u : 0x05040100u);
            }
            *reinterpret_cast<uint4*>(wt + (col + m) * ld + r0) = make_uint4(t[0], t[1], t[2], t[3]);
        }
        return there;
    }
    eight_rows(P, r0, col, trits_of, [&](int i, int m, float x) {
        const uint32_t b = half_bits<HT>(__is_same(HT, _Float16) ? x * by : x);
        v[m][i >> 1] = (i & 1) != 0 ? v[m][i >> 1] | b << 16 : b;
    });
#pragma unroll
    for (int m = 0; m < 8; ++m) {
        *reinterpret_cast<uint4*>(wt + (col + m) * ld + r0) = make_uint4(v[m][0], v[m][1], v[m][2], v[m][3]);
        there |= ((v[m][0] | v[m][1] | v[m][2] | v[m][3]) & 0x7fff7fffu) != 0u ? 1u << m : 0u;
    }
    return there;
}

// The largest finite magnitude that the weights of a row's group can have, and the power of two that brings magnitudes up to `most` below 2^15 (1 where
// there are none), itself within fp32's normal numbers.
__device__ __forceinline__ float finite_max(float m, float x) { return isfinite(x) && fabsf(x) > m ? fabsf(x) : m; }
__device__ __forceinline__ float affine_top(const PackArgs& P, int a, int64_t g) {
    const float s = P.scale[g], o = a >= 5 ? 0.0f : P.offset[g];
    const float L = a == 1 ? 255.0f : (a == 2 ? 15.0f : (a == 3 ? 7.0f : (a == 4 ? 3.0f : 1.0f)));
    const float top = isfinite(s) ? fminf(fabsf(fmaf(s, L, o)), 3.40282347e38f) : 0.0f;       // codes that are there may be smaller ones than L
    return isfinite(o) ? fmaxf(fabsf(o), top) : 0.0f;
}
// half_lost of each weight of a group: no more than half a step and than the largest.  From HALF_GROUP on a group's weights are off by 2^-15 of its largest at most, and nothing
// counts as lost.
constexpr float HALF_GROUP = 0x1p-10f;
__device__ __forceinline__ float group_lost(const PackArgs& P, int a, int64_t g, float by) {
    const float top = affine_top(P, a, g);
    return top > 0.0f && top * by < HALF_GROUP ? fmaxf(fminf(top * by, 0x1p-25f), 0x1p-100f) * 0x1p25f : 0.0f;
}
// A row's group's part in the largest magnitude and in the smallest, weights that stay as they are counting 16 times: HALF_GROUP is 16 HALF_NORMAL.
__device__ __forceinline__ void group_range(const PackArgs& P, int64_t row, int64_t j, float& most, float& least, bool& coded) {
    const int64_t rb = row / P.R_u, u = rb * P.n_chunks + j;
    int64_t base;
    const int a = pk_action(P, u, base);
    if (a == 0) {
#pragma unroll 2
        for (int32_t c = 0; c < P.G; c += 8) {
            float w[8];
            skip_row(P, row, j * P.G + c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                most = finite_max(most, w[i]);
                least = w[i] != 0.0f ? fminf(least, 16.0f * fabsf(w[i])) : least;
            }
        }
        return;
    }
    const float top = affine_top(P, a, u * P.R_u + row - rb * P.R_u);
    most = fmaxf(most, top);
    least = top > 0.0f ? fminf(least, top) : least;
    coded |= top > 0.0f;
}
// Of eight rows from r0 on, those that rounding takes something from in an octet of columns.
__device__ __forceinline__ int32_t rows_lost(const PackArgs& P, int64_t r0, int64_t col, float by) {
    const int64_t j = col / P.G;
    int32_t n = 0;
#pragma unroll 1
    for (int64_t row = r0; row < r0 + 8 && row < P.rows; ++row) {
        const int64_t rb = row / P.R_u, u = rb * P.n_chunks + j;
        int64_t base;
        const int a = pk_action(P, u, base);
        float lost = 0.0f;
        if (a == 0) {
            float w[8];
            skip_row(P, row, col, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) lost += half_lost(w[i], w[i] * by);
        } else {
            lost = group_lost(P, a, u * P.R_u + row - rb * P.R_u, by);
        }
        n += lost > 0.0f ? 1 : 0;
    }
    return n;
}
__device__ __forceinline__ float power_below(float most) {
    const int e = (int)(__float_as_uint(most) >> 23);       // biased; most < 2^(e - 126)
    const int by = most > 0.0f ? 127 + 14 - (e - 127) : 127;
    return __uint_as_float((uint32_t)(by > 253 ? 253 : by) << 23);
}

#endif  // __HIPCC__

}  // namespace windq
