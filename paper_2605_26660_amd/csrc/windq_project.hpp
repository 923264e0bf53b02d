// What the products of a packed plan with many tokens share: the packed matrix as the kernels see it, codes as matrix
// operands, adapters, grouping of tokens by adapter.
//
// A group's reconstruction is affine in its codes, w_hat = offset + scale * code, so
//     sum_c w_hat x_c = scale * sum_c f_c x_c + beta * sum_c x_c,    f = code + f0,  beta = offset - f0 * scale
// and the sum over f needs no rounded weight: f is a small number that bfloat16 holds exactly.  f0 is chosen so that f comes out of
// a code's bits by one shift and one and-or for two of them: with b code bits below the leading one of a bfloat16 mantissa,
// 2^b + code has the bit pattern of 2^b with the code or-ed in.
//     8 bits  code         (0 .. 255, converted)    4 bits  16 + code     3 bits  8 + code     2 bits  4 + code
//     1.58    4 + trit, beta = -5 scale             1 bit   +-1, beta = 0                       skip    the weight, scale 1
// f is off centre by up to five times its spread, which costs two to three bits of the fp32 sum over one chunk: nothing to an output of
// bfloat16.  For fp32 activations f is brought to its centre first (q - 7.5 and the like: still exact in bfloat16).
#pragma once

#include "windq_common.hpp"

namespace windq {

struct PackArgs {
    const void* W;
    int64_t ld;
    int32_t w_f32;             // W holds fp32
    const uint8_t* mask;       // or null
    int64_t mask_ld;
    const uint8_t* action;
    const int64_t* code_off;
    const uint8_t* codes;
    int64_t codes_bytes;
    const float* scale;
    const float* offset;
    int64_t rows, cols, R_u;
    int32_t G, n_chunks;
};

struct AdapterArgs {
    const void* a;             // [n][max_rank][cols]
    const void* b;             // [n][rows][max_rank]
    const float* alpha;        // or null
    const int32_t* rank;       // or null
    const int32_t* of;         // [tokens]
    int32_t n, max_rank;
};

int check_packed(const windq_packed* P, PackArgs* A);
int check_adapters(const windq_adapters* ad, const int32_t* adapter_of, int32_t dtype, AdapterArgs* A);

#ifdef __HIPCC__

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ bf16x8 as_bf16x8(uint4 v) { return __builtin_bit_cast(bf16x8, v); }

__device__ __forceinline__ uint32_t f32_to_bf16_bits(float x) {
    const __bf16 b = (__bf16)x;                            // to nearest, ties to even, NaN kept
    return (uint32_t)__builtin_bit_cast(uint16_t, b);
}

// x as three bfloat16 terms that add up to it (24 bits of mantissa).  What is not finite is its first term alone.  Finite values that would round
// to infinity, from 2^128 - 2^119 on, have bfloat16's largest one for their first term.
__device__ __forceinline__ void split3(float x, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
    hi = f32_to_bf16_bits(x) - ((__float_as_uint(x) & 0x7fff8000u) == 0x7f7f8000u ? 1u : 0u);
    float r = x - bf16_bits_to_f32(hi);
    const bool fine = (__float_as_uint(r) & 0x7f800000u) != 0x7f800000u;      // x is finite
    r = fine ? r : 0.0f;
    mid = f32_to_bf16_bits(r);
    lo = f32_to_bf16_bits(r - bf16_bits_to_f32(mid));
}

__device__ __forceinline__ int adapter_rank(const AdapterArgs& A, int k) {
    const int r = A.rank != nullptr ? A.rank[k] : A.max_rank;
    return r < 0 ? 0 : (r > A.max_rank ? A.max_rank : r);
}

__device__ __forceinline__ int64_t pk_bytes_per_group(int a, int G) {
    switch (a) {
        case 1: return G;
        case 2: return G >> 1;
        case 3: return (G * 3) >> 3;
        case 4: return G >> 2;
        case 5: return (G + 4) / 5;
        case 6: return G >> 3;
        default: return 0;
    }
}

// The treatment of unit u and where its codes start; an entry that does not fit counts as skip.
__device__ __forceinline__ int pk_action(const PackArgs& P, int64_t u, int64_t& base) {
    int a = P.action[u];
    base = P.code_off[u];
    if (a >= WINDQ_N_ACTIONS) a = 0;
    if (a != 0 && (base < 0 || (base & 15) != 0 || base > P.codes_bytes - pk_bytes_per_group(a, P.G) * P.R_u)) a = 0;
    return a;
}

// f0, and what f comes down by when it is centred.
__device__ __forceinline__ float pk_f0(int a) { return a == 2 ? 16.0f : (a == 3 ? 8.0f : (a == 4 ? 4.0f : (a == 5 ? 5.0f : 0.0f))); }
__device__ __forceinline__ float pk_centre(int a) { return a == 1 ? 127.5f : (a == 2 ? 23.5f : (a == 3 ? 11.5f : (a == 4 ? 5.5f : (a == 5 ? 5.0f : 0.0f)))); }

// beta = offset - f0 * scale (1.58 and 1 bit have no offset of their own).
__device__ __forceinline__ void pk_affine(int a, float scale, float offset, bool centred, float& alpha, float& beta) {
    alpha = a == 0 ? 1.0f : scale;
    const float o = a >= 5 || a == 0 ? 0.0f : offset;
    const float f0 = centred ? pk_f0(a) - pk_centre(a) : pk_f0(a);
    beta = a == 0 ? 0.0f : o - f0 * scale;
}
__device__ __forceinline__ uint32_t centred_pair(uint32_t v, float c) {
    return __builtin_amdgcn_perm(__float_as_uint(__uint_as_float(v & 0xffff0000u) - c), __float_as_uint(__uint_as_float(v << 16) - c), 0x07060302u);
}
__device__ __forceinline__ uint4 centred(uint4 f, float c) { return make_uint4(centred_pair(f.x, c), centred_pair(f.y, c), centred_pair(f.z, c), centred_pair(f.w, c)); }

// Two copies of v side by side, kept from the compiler: it would make one multiplication (16 clocks) of this and the shift that follows.
__device__ __forceinline__ uint32_t twice(uint32_t v, int by, uint32_t with) {
    uint32_t t = v << by | with;
    asm("" : "+v"(t));
    return t;
}

// Eight 2-bit fields (16 bits of v) as 4 + field.
__device__ __forceinline__ uint4 fields2(uint32_t v) {
    const uint32_t t = twice(v, 14, v);                    // fields 2i and 2i + 1 at bits 4i and 4i + 16
    uint4 f;
    f.x = ((t << 5) & 0x00600060u) | 0x40804080u;
    f.y = ((t << 1) & 0x00600060u) | 0x40804080u;
    f.z = ((t >> 3) & 0x00600060u) | 0x40804080u;
    f.w = ((t >> 7) & 0x00600060u) | 0x40804080u;
    return f;
}

// Eight signs (8 bits of v): bit 1 is +1, bit 0 is -1.
__device__ __forceinline__ uint4 fields1(uint32_t v) {
    const uint32_t n = ~v;
    const uint32_t t = twice(n, 15, n & 0xffu);            // bits 2i and 2i + 1 at 2i and 2i + 16
    uint4 f;
    f.x = ((t << 15) & 0x80008000u) | 0x3f803f80u;
    f.y = ((t << 13) & 0x80008000u) | 0x3f803f80u;
    f.z = ((t << 11) & 0x80008000u) | 0x3f803f80u;
    f.w = ((t << 9) & 0x80008000u) | 0x3f803f80u;
    return f;
}

// Eight 4-bit fields as 16 + field.
__device__ __forceinline__ uint4 fields4(uint32_t v) {
    const uint32_t e = twice(v, 12, v & 0xffffu), o = twice(v >> 16, 12, v >> 16);   // fields 2i and 2i + 1 at bits 8i and 8i + 16
    uint4 f;
    f.x = ((e << 3) & 0x00780078u) | 0x41804180u;
    f.y = ((e >> 5) & 0x00780078u) | 0x41804180u;
    f.z = ((o << 3) & 0x00780078u) | 0x41804180u;
    f.w = ((o >> 5) & 0x00780078u) | 0x41804180u;
    return f;
}

// Eight 3-bit fields (24 bits of v) as 8 + field.
__device__ __forceinline__ uint4 fields3(uint32_t v) {
    uint4 f;
    f.x = ((v << 4) & 0x70u) | ((v << 17) & 0x700000u) | 0x41004100u;
    f.y = ((v >> 2) & 0x70u) | ((v << 11) & 0x700000u) | 0x41004100u;
    f.z = ((v >> 8) & 0x70u) | ((v << 5) & 0x700000u) | 0x41004100u;
    f.w = ((v >> 14) & 0x70u) | ((v >> 1) & 0x700000u) | 0x41004100u;
    return f;
}

// Eight bytes as numbers 0 .. 255.
__device__ __forceinline__ uint32_t bytes_pair(uint32_t v, int lo) {
    const float a = (float)((v >> (8 * lo)) & 0xffu), b = (float)((v >> (8 * lo + 8)) & 0xffu);
    return __float_as_uint(a) >> 16 | (__float_as_uint(b) & 0xffff0000u);
}
__device__ __forceinline__ uint4 fields8(uint32_t v0, uint32_t v1) {
    return make_uint4(bytes_pair(v0, 0), bytes_pair(v0, 2), bytes_pair(v1, 0), bytes_pair(v1, 2));
}

// Entry b of the table that turns a byte into its five trits, as five 2-bit fields.
__device__ __forceinline__ uint32_t trit_fields(uint32_t b) {
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        t |= (b % 3u) << (2 * i);
        b /= 3u;
    }
    return t;
}

// The eight trits of octet o of a row, as 2-bit fields.
__device__ __forceinline__ uint32_t octet_trits(const uint8_t* __restrict__ row, int o, const uint16_t* __restrict__ trits_of) {
    const uint32_t first = (uint32_t)o * 8u, k = first / 5u, r = first - k * 5u;
    uint32_t v = (uint32_t)trits_of[row[k]] | (uint32_t)trits_of[row[k + 1]] << 10;
    if (r > 2u) v |= (uint32_t)trits_of[row[k + 2]] << 20;                    // trits r .. r + 7 reach the third byte
    return v >> (2 * r);
}

// Octet o of a group as eight f, from the group's first byte.  Any width of chunk, any alignment, treatment lane by lane (not skip).
__device__ __forceinline__ uint4 octet_fields(int a, const uint8_t* __restrict__ row, int o, const uint16_t* __restrict__ trits_of) {
    switch (a) {
        case 1: {
            uint32_t v[2];
            __builtin_memcpy(v, row + o * 8, 8);
            return fields8(v[0], v[1]);
        }
        case 2: {
            uint32_t v;
            __builtin_memcpy(&v, row + o * 4, 4);
            return fields4(v);
        }
        case 3: {
            const uint8_t* p = row + o * 3;
            return fields3((uint32_t)p[0] | (uint32_t)p[1] << 8 | (uint32_t)p[2] << 16);
        }
        case 4: {
            uint16_t v;
            __builtin_memcpy(&v, row + o * 2, 2);
            return fields2(v);
        }
        case 5: return fields2(octet_trits(row, o, trits_of) & 0xffffu);
        default: return fields1(row[o]);
    }
}

// The code of column c of a group (skip excluded), and its weight in fp64.
__device__ __forceinline__ double pk_weight(int a, const uint8_t* __restrict__ row, int c, float scale, float offset) {
    uint32_t q;
    switch (a) {
        case 1: q = row[c]; break;
        case 2: q = (row[c >> 1] >> (4 * (c & 1))) & 15u; break;
        case 3: {
            const int bit = 3 * c;
            const uint32_t v = (uint32_t)row[bit >> 3] | ((bit & 7) > 5 ? (uint32_t)row[(bit >> 3) + 1] << 8 : 0u);
            q = (v >> (bit & 7)) & 7u;
            break;
        }
        case 4: q = (row[c >> 2] >> (2 * (c & 3))) & 3u; break;
        case 5: {
            uint32_t v = row[c / 5];
            for (int i = c % 5; i > 0; --i) v /= 3u;
            return (double)scale * ((double)(v % 3u) - 1.0);
        }
        default: return ((row[c >> 3] >> (c & 7)) & 1u) != 0u ? (double)scale : -(double)scale;
    }
    return fma((double)q, (double)scale, (double)offset);
}

__device__ __forceinline__ float elem(const void* p, int64_t i, bool f32) {
    return f32 ? static_cast<const float*>(p)[i] : bf16_bits_to_f32(static_cast<const uint16_t*>(p)[i]);
}

// w_hat[row] . x weight by weight in fp64: what a result that did not come out finite is formed by again.  It ends at the first
// column that makes it NaN.
template <typename XT>
__device__ __forceinline__ double pk_slow_dot(const PackArgs& P, int64_t row, const XT* __restrict__ x) {
    const int64_t rb = row / P.R_u, lrow = row - rb * P.R_u;
    double sum = 0.0;
    for (int j = 0; j < P.n_chunks && sum == sum; ++j) {
        const int64_t u = rb * P.n_chunks + j;
        int64_t base;
        const int a = pk_action(P, u, base);
        const int64_t g = u * P.R_u + lrow;
        const uint8_t* r = P.codes + base + lrow * pk_bytes_per_group(a, P.G);
        const float s = P.scale[g], o = P.offset[g];
        for (int c = 0; c < P.G && sum == sum; ++c) {
            const int64_t col = (int64_t)j * P.G + c;
            if (a != 0 && P.mask != nullptr && ((P.mask[row * P.mask_ld + (col >> 3)] >> (col & 7)) & 1u) != 0u) continue;
            const double w = a == 0 ? (double)elem(P.W, row * P.ld + col, P.w_f32 != 0) : pk_weight(a, r, c, s, o);
            double xv;
            if constexpr (sizeof(XT) == 4) xv = (double)x[col];
            else xv = (double)bf16_bits_to_f32(x[col]);
            sum = fma(w, xv, sum);
        }
    }
    return sum;
}

// Protection bits of an octet as a mask over eight bfloat16 values (all ones where the weight is kept).
__device__ __forceinline__ uint4 keep_words(uint32_t m) {
    const uint32_t k = ~m;
    uint4 w;
    w.x = ((k & 1u) != 0u ? 0xffffu : 0u) | ((k & 2u) != 0u ? 0xffff0000u : 0u);
    w.y = ((k & 4u) != 0u ? 0xffffu : 0u) | ((k & 8u) != 0u ? 0xffff0000u : 0u);
    w.z = ((k & 16u) != 0u ? 0xffffu : 0u) | ((k & 32u) != 0u ? 0xffff0000u : 0u);
    w.w = ((k & 64u) != 0u ? 0xffffu : 0u) | ((k & 128u) != 0u ? 0xffff0000u : 0u);
    return w;
}
__device__ __forceinline__ uint4 and4(uint4 a, uint4 b) { return make_uint4(a.x & b.x, a.y & b.y, a.z & b.z, a.w & b.w); }

// Eight skip weights, term 0 (bfloat16, or the first of fp32's three), 1 or 2.
__device__ __forceinline__ uint4 skip_octet(const PackArgs& P, int64_t row, int64_t col, int term) {
    if (P.w_f32 == 0) {
        if (term > 0) return make_uint4(0u, 0u, 0u, 0u);
        return *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(P.W) + row * P.ld + col);
    }
    const float* p = static_cast<const float*>(P.W) + row * P.ld + col;
    uint32_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t t[3];
        split3(p[j], t[0], t[1], t[2]);
        v[j] = term == 0 ? t[0] : (term == 1 ? t[1] : t[2]);
    }
    return make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}

#endif  // __HIPCC__

}  // namespace windq
