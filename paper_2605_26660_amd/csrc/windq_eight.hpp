// Products of 8-bit tokens with a packed plan: the tokens' and the plan's forms, and what their kernels share.
//
// A token is x_c = sigma q_c with integers q_c of eight bits; a group's weights are w_c = alpha f_c + beta with f_c its code, or the code less 128
// where it has eight bits.  So
//     sum_c w_c x_c = sigma * sum over chunks of (alpha * sum_c f_c q_c + beta * sum_c q_c)
// and both sums over a chunk are exact in 32-bit integers (512 columns x 128 x 127 at most): the matrix instructions multiply codes as they are, at
// twice the rate of bfloat16, and a code needs no more unpacking than a shift and a mask of four at a time.
//     8 bits  code - 128, beta = offset + 128 scale     4, 3 and 2 bits  code, beta = offset
//     1.58    trit 0 .. 2, beta = -scale                1 bit            bit 0 or 1, alpha = 2 scale, beta = -scale
//
// A chunk's columns are cut into k-blocks of 32 S columns, S <= 4 alike; where they do not come out even the last one is filled with zeros, in
// the tokens and in the plan.  In a step of 32 columns the lower half of a wavefront's lanes takes the first 16 of them, the upper half the others.
#pragma once

#include "windq_act.hpp"
#include "windq_adapters.hpp"

namespace windq {

constexpr int EIGHT_ROWS = 32;                             // rows of a row block: the M side of 32x32x32 instructions

struct EightShape {
    int64_t rows, cols, R_u;
    int32_t G, n_chunks;
    int32_t S, per_chunk;      // steps of a k-block, k-blocks of a chunk
    int32_t n_kb;
    int64_t width, sums_ld;    // bytes of a token, sums of a token (in fours)
    int64_t RB;                // row blocks of a unit
    int64_t n_rb, NB;          // unit row blocks; row blocks of the matrix
    int64_t U, affine, header; // units; bytes ahead of alpha and beta, and of the fields
};

// How a chunk is cut: as few k-blocks as have four steps at most, alike.
inline void eight_cut(int32_t G, int32_t* S, int32_t* per_chunk) {
    const int32_t steps = (G + 31) / 32;
    *per_chunk = (steps + 3) / 4;
    *S = (steps + *per_chunk - 1) / *per_chunk;
}

// The serving form's first part, of the matrix's row blocks (unit by unit down the rows) and k-blocks: a word each, of where its fields begin in
// 256s of bytes and of their kind (the lowest three bits); then the 32 rows' alpha and beta, again for each k-block of a chunk.
inline EightShape eight_shape(int64_t rows, int64_t cols, int64_t R_u, int32_t G) {
    EightShape E;
    E.rows = rows;
    E.cols = cols;
    E.R_u = R_u;
    E.G = G;
    E.n_chunks = (int32_t)(cols / G);
    eight_cut(G, &E.S, &E.per_chunk);
    E.n_kb = E.n_chunks * E.per_chunk;
    E.width = (int64_t)E.n_kb * E.S * 32;
    E.sums_ld = ((int64_t)E.n_kb + 3) / 4 * 4;
    E.RB = (R_u + EIGHT_ROWS - 1) / EIGHT_ROWS;
    E.n_rb = rows / R_u;
    E.NB = E.n_rb * E.RB;
    E.U = E.n_rb * E.n_chunks;
    E.affine = (int64_t)round_up((size_t)(E.NB * E.n_kb) * 4, 256);
    E.header = E.affine + E.NB * E.n_kb * 256;
    return E;
}

// Kinds of fields: 0 weights that stay as they are, 1: 8 bits, 2: 4 bits (3 as well), 3: nothing (zeros), 4: 2 bits (trits as well), 6: 1 bit.
constexpr int EIGHT_NOTHING = 3;
__host__ __device__ inline int eight_kind(int action) { return action == 3 ? 2 : (action == 5 ? 4 : action); }

// Bytes of a row block's fields of one k-block: a string of words a lane, step by step, in pieces of 16 bytes, [piece][lane][16], and what is left over,
// [lane][the rest].  8 bits: four words a step, 4 bits: two, 2 bits: one, 1 bit: one for two steps.  A word's four bytes hold columns 4 i + (0 .. 3)
// at bits b i of each byte, b bits a field: w >> b i, masked, are four operands of the matrix instruction.
//   Weights that stay as they are: [step][term][half of its 16 columns][lane][8 bfloat16], one term, or three where they are fp32.
__host__ __device__ inline int64_t eight_bytes(int kind, int S, bool w_f32) {
    switch (kind) {
        case 0: return (w_f32 ? 6144 : 2048) * (int64_t)S;
        case 1: return 1024 * (int64_t)S;
        case 2: return 512 * (int64_t)S;
        case 4: return 256 * (int64_t)S;
        case 6: return 256 * (int64_t)((S + 1) / 2);
        default: return 0;
    }
}

// Bytes of a lane's string.
__host__ __device__ inline int eight_string(int kind, int S) { return kind == 1 ? 16 * S : (kind == 2 ? 8 * S : (kind == 4 ? 4 * S : 4 * ((S + 1) / 2))); }
constexpr int EIGHT_PAST = 256;                            // bytes past its last fields that an image has: a lane reads whole pieces

constexpr int64_t EIGHT_MOST = (int64_t)1 << 37;           // bytes of an image: 256s of them in 29 bits of a word

struct EightPlan {
    const char* image;
    int64_t bytes;
    int64_t header;
};

struct EightArgs {
    EightPlan P[2];            // gate and up, or one
    const int8_t* codes;
    const float* scale;
    const int32_t* sums;
    int64_t T;
    void* Y;
    int64_t ldy;
    int64_t R_u, RB, NB, width, sums_ld, affine;            // affine: where alpha and beta begin
    int32_t n_kb, act, w_f32;
};

#ifdef __HIPCC__

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ i32x4 as_i32x4(uint4 v) { return __builtin_bit_cast(i32x4, v); }

// Where a row block's fields of a k-block lie and what they are.  What does not lie between the header and the image's end counts as
// nothing, whatever the image's words say.
struct EightBlock {
    const char* fields;
    int kind;
};
__device__ __forceinline__ uint32_t eight_word(const EightPlan& P, uint32_t word, int S, bool w_f32) {
    const int64_t at = (int64_t)(word >> 3) << 8;
    const int kind = (int)(word & 7u);
    return kind != EIGHT_NOTHING && at >= P.header && at <= P.bytes - EIGHT_PAST - eight_bytes(kind, S, w_f32) ? word : (uint32_t)EIGHT_NOTHING;
}
__device__ __forceinline__ EightBlock eight_block(const EightPlan& P, uint32_t word) { return {P.image + ((uint64_t)(word >> 3) << 8), (int)(word & 7u)}; }

// Operands of a step out of a lane's words.
__device__ __forceinline__ i32x4 eight_fields4(uint2 v) {
    i32x4 f;
    f[0] = (int)(v.x & 0x0f0f0f0fu);
    f[1] = (int)((v.x >> 4) & 0x0f0f0f0fu);
    f[2] = (int)(v.y & 0x0f0f0f0fu);
    f[3] = (int)((v.y >> 4) & 0x0f0f0f0fu);
    return f;
}
// A lane's string of one row block and k-block.
template <int S>
struct EightFields {
    uint32_t v[S][4];
    __device__ __forceinline__ void load(int kind, const char* __restrict__ fields, int lane) {
        auto piece = [&](int k, int stride) { __builtin_memcpy(v[k], fields + k * 1024 + lane * stride, 16); };
        // The first piece whatever the kind (what holds no string reads its first bytes), so that no register waits for what comes in by another
        // way; a lane's stride in it by kind, a byte each.
        constexpr uint64_t strides = 16ull << 8 | (S == 1 ? 8ull : 16ull) << 16 | (uint64_t)(4 * S) << 32 | (uint64_t)(4 * ((S + 1) / 2)) << 48;
        piece(0, (int)(strides >> (8 * kind)) & 0xff);
        if constexpr (S > 1) {
            if (kind == 1 || (S > 2 && kind == 2)) {
                piece(1, kind == 2 && S == 3 ? 8 : 16);
                if constexpr (S > 2) {
                    if (kind == 1) {
                        piece(2, 16);
                        if constexpr (S == 4) piece(3, 16);
                    }
                }
            }
        }
    }
    __device__ __forceinline__ uint32_t word(int k) const { return v[k >> 2][k & 3]; }
    // The operands of all steps; zeros for what holds no string.  1 and 2 bits (nine weights of ten in a plan of two bits on average) by the same instructions: a branch
    // costs more than they do.
    __device__ __forceinline__ void operands(int kind, i32x4 (&w)[S]) const {
        if ((kind & 4) != 0) {
            const bool one = kind == 6;
            const uint32_t mask = one ? 0x01010101u : 0x03030303u;
            const int by = one ? 1 : 2;
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const uint32_t f = one ? word(s >> 1) >> (4 * (s & 1)) : word(s);
#pragma unroll
                for (int i = 0; i < 4; ++i) w[s][i] = (int)((f >> (i * by)) & mask);
            }
        } else if (kind == 2) {
#pragma unroll
            for (int s = 0; s < S; ++s) w[s] = eight_fields4(make_uint2(word(2 * s), word(2 * s + 1)));
        } else if (kind == 1) {
#pragma unroll
            for (int s = 0; s < S; ++s) w[s] = as_i32x4(make_uint4(v[s][0], v[s][1], v[s][2], v[s][3]));
        } else {
#pragma unroll
            for (int s = 0; s < S; ++s) w[s] = i32x4{};
        }
    }
};

// All loads done, direct ones among them.  As a builtin: the compiler then knows it of its own loads and waits for none of them again, which would wait for
// direct loads that it does not count.
__device__ __forceinline__ void wait_for_loads() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0f70);
    asm volatile("" ::: "memory");
}

// Eight of a token's integers as bfloat16: exact.
__device__ __forceinline__ bf16x8 eight_as_bf16(uint32_t a, uint32_t b) {
    auto pair = [](uint32_t v, int lo) {
        const float x = (float)(int)(int8_t)(v >> (8 * lo)), y = (float)(int)(int8_t)(v >> (8 * lo + 8));
        return __float_as_uint(x) >> 16 | (__float_as_uint(y) & 0xffff0000u);
    };
    return as_bf16x8(make_uint4(pair(a, 0), pair(a, 2), pair(b, 0), pair(b, 2)));
}

__device__ __forceinline__ void eight_store(float* p, float v) { *p = v; }
__device__ __forceinline__ void eight_store(uint16_t* p, float v) { *p = (uint16_t)f32_to_bf16_bits(v); }

#endif  // __HIPCC__

}  // namespace windq
