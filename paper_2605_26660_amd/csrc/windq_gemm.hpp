// dX = w_hat^T dY in bfloat16: a plain product of two matrices whose rows lie along the sum's axis.
//
// Codes lie along columns and the sum runs along rows, so a tile of weights would have to be turned for every 128 tokens.  The packed
// matrix is reconstructed once instead, rounded to bfloat16 and turned (wt [cols][rows], 2 bytes a weight; 29 to 33 of 289 us at 2048 tokens through
// 11008 x 4096; for one token too: 4096 x 4096 45 us, 373 with tiles turned on the way), and the product then spends nothing but matrix instructions and their operands' way (160 us, 1160 TFLOP/s).
// That rounding is of the weights alone and once: dX is 2.4e-3 off the formula in 64 bits (norm by norm) where its own rounding to bfloat16 alone would make it 1.7e-3.  Two terms of a
// weight would undo it for twice the matrix instructions; a caller who needs it passes fp32, where nothing is rounded.
//   256 columns x 128 tokens a workgroup, four wavefronts with 128 x 64 results each as 4 x 2 fragments of 32x32x16 instructions, one per SIMD; 128 columns where
// that would leave CUs without a workgroup.
//   64 of the sum at a time go to LDS by direct loads, three buffers: while one is multiplied the next has landed and the one
// after is on its way.  There is one barrier per buffer, ahead of its last step: by then all of it has been read into registers, and the next
// one's first operands are read across it.  A row's eight 16-byte slots are exchanged by the bits above the row's lowest, so that sixteen
// lanes reading sixteen rows' same slot meet all 64 banks (two rows have a turn of them).
#pragma once

#include "windq_pair.hpp"

namespace windq {

constexpr int GM_MOST = 256, GM_N = 128, GM_K = 64, GM_THREADS = 256, GM_BUFFERS = 3;

// What dX is formed from again, column by column: the caller's.
struct AgainArgs {
    const uint16_t* dH;
    const uint16_t* G;
    const uint16_t* U;
    int64_t ld_dh, ld_save;
};

struct GemmArgs {
    const uint16_t* wt;        // [cols rounded up to GM_MOST][K]
    const uint16_t* dY;        // [T][ldy], zeros from rows to K
    int64_t ldy;
    int32_t K;                 // rows rounded up to GM_K
    int64_t T, cols;
    uint16_t* dX;
    int64_t ldx;
    const float* dh;           // or null: no adapters
    const uint16_t* at;        // [n][cols][max_rank]
    AdapterArgs A;
    uint32_t col_blocks;
    float* part;               // [splits][T][cols] sums over a part of the rows, or null: one workgroup has them all
    int32_t tiles, each;       // workgroups of a split, its steps of GM_K
    const float* by_token;     // halves: the powers of two that a token's results are multiplied by, and an octet of columns'
    const float* by_octet;
    // Of a pair (windq_gated) `columns` are rows of the gate and of the up, 32 and 32 in turn, and dX is H.
    PackArgs gate;
    PairArgs pair;
    const float* by_row;       // the powers of those rows, and as in by_token what rounding has taken from them (with_loss)
    const uint16_t* raw;       // the caller's X
    int64_t ld_raw;
    // Of its way back: weights of an octet of columns that rounding has taken something from, by 2^-25 at most.
    const int32_t* lost_octet;
    const uint32_t* there_octet;   // its columns that have something other than 0 where there are no codes or a mask lies over them: with no weight lost the others' results are 0
    AgainArgs again;
};

inline int64_t gemm_k(int64_t rows) { return (rows + GM_K - 1) / GM_K * GM_K; }
// Where 128-column tiles are fewer than the CUs the sum is split over workgroups, four steps or more each, and another kernel joins the
// parts in order and adds the adapters': 11008 x 4096, 64 tokens (32 tiles) 109 -> 70 us, 4096 x 4096, 1 token 59 -> 45.
constexpr int GM_TILES = 256, GM_LEAST = 4;
inline int32_t gemm_each(int64_t K, int64_t tiles) {
    const int64_t steps = K / GM_K, most = tiles < GM_TILES ? GM_TILES / tiles : 1, each = (steps + most - 1) / most;
    return (int32_t)(each > GM_LEAST ? each : GM_LEAST);
}
// Most floats of the parts, for so many tokens or fewer.
inline int64_t gemm_parts(int64_t T, int64_t K, int64_t cols) {
    const int64_t all = (int64_t)GM_TILES * 128 * GM_N, splits = (K / GM_K + GM_LEAST - 1) / GM_LEAST;
    return T * cols * splits < all ? T * cols * splits : all;
}
inline int64_t gemm_cols(int64_t cols) { return (cols + GM_MOST - 1) / GM_MOST * GM_MOST; }

#ifdef __HIPCC__

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Of a power of two.  Two of them are put on by their exponents: their product, or a result times the first, may lie outside fp32 where the result does not.
__device__ __forceinline__ int exponent_of(float power) { return (int)((__float_as_uint(power) >> 23) & 0xffu) - 127; }

// What half precision takes from a value x that enters as y, x times a power of two: y below its normal numbers (2^-14) is rounded to a multiple of 2^-24, which may
// be all of it.  A factor of the product is below 2^15, so that a sum is off by 2^15 of what is lost; times 2^25: the results, as they come out of the product, for which
// that is 2^-10 and more.  One below what its token and its row have lost is formed again weight by weight.
constexpr float HALF_NORMAL = 0x1p-14f;
__device__ __forceinline__ float half_lost(float x, float y) {
    const float off = fabsf(y) < HALF_NORMAL && x != 0.0f ? fmaxf(fabsf(y - (float)(_Float16)y), y == 0.0f ? 0x1p-100f : 0.0f) : 0.0f;
    return off * 0x1p25f;
}
// A power of two with a loss in its last sixteen bits: the loss as bfloat16, rounded up.  Whoever reads the power reads its exponent.  Where there is nothing but zeros, and
// nothing to lose, the loss is far below 0, whatever the other side adds.
__device__ __forceinline__ float with_loss(float power, float lost) { return __uint_as_float(__float_as_uint(power) | (__float_as_uint(lost) + 0xffffu) >> 16); }
__device__ __forceinline__ float loss_in(float word) { return __uint_as_float(__float_as_uint(word) << 16); }
// The bit above them: a chunk of columns with codes that stand for something other than 0.
__device__ __forceinline__ float with_codes(float power, bool codes) { return __uint_as_float(__float_as_uint(power) | (codes ? 0x10000u : 0u)); }
__device__ __forceinline__ bool has_codes(float word) { return (__float_as_uint(word) & 0x10000u) != 0u; }
__device__ __forceinline__ float power_of_nothing() { return __uint_as_float(0x0000ff7fu); }

// A kernel's first argument from where it lies, for what is seldom needed: the compiler would load all of it at the kernel's start, into more scalar registers than there are.
template <typename Args>
__device__ __forceinline__ const Args& argument_in_place() {
    typedef const __attribute__((address_space(4))) Args* Place;
    Place at = (Place)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    return *(const Args*)at;
}

// Results of a token and an octet of columns below which what both have lost counts.
__device__ __forceinline__ float lost_below(float by_token, float by_octet, int32_t lost) { return loss_in(by_token) + loss_in(by_octet) + (float)lost; }

// Eight columns of dX of a token in fp64, by all lanes of a wavefront, ROWS times 64 rows at a time: all of them get the sums.  Two rounds of loads a turn, without branches between
// those of a round; 240 us for 11008 rows, where one load after the other takes 480.  Seldom: none of 8.4 M values at G of 1.7 on average, two to four at 8, where
// most slopes are 0.  WINDOW: code streams of eight bytes and more, read eight at a time.
template <int ROWS, bool WINDOW>
__device__ __forceinline__ void dx_again_by(const PackArgs& gate, const PackArgs& up, int act, const AgainArgs& A, int64_t t, int64_t col, int lane, double (&sum)[8]) {
    const uint32_t j = (uint32_t)(col / gate.G), o = (uint32_t)(col - (int64_t)j * gate.G) >> 3, R_u = (uint32_t)gate.R_u, n_rows = (uint32_t)gate.rows;
#pragma unroll
    for (int m = 0; m < 8; ++m) sum[m] = 0.0;
#pragma unroll 1
    for (uint32_t row0 = 0; row0 < n_rows; row0 += 64 * ROWS) {
        uint32_t row[ROWS], rb[ROWS], action[2][ROWS];
        uint16_t h[ROWS], g[ROWS], u[ROWS];
        int64_t base[2][ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const uint32_t r = row0 + 64 * i + lane;
            row[i] = r < n_rows ? r : n_rows - 1;
            rb[i] = row[i] / R_u;
            h[i] = A.dH[t * A.ld_dh + row[i]];
            g[i] = A.G[t * A.ld_save + row[i]];
            u[i] = A.U[t * A.ld_save + row[i]];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const PackArgs& P = k == 0 ? gate : up;
                action[k][i] = P.action[(int64_t)rb[i] * P.n_chunks + j];
                base[k][i] = P.code_off[(int64_t)rb[i] * P.n_chunks + j];
            }
        }
        int kind[2][ROWS];
        float s[2][ROWS], offset[2][ROWS];
        uint64_t v[2][ROWS];
        uint4 kept[2][ROWS][2];
        uint8_t mask[2][ROWS];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                const PackArgs& P = k == 0 ? gate : up;
                const uint32_t lrow = row[i] - rb[i] * R_u;
                // as pk_action has it
                const int a = action[k][i] < WINDQ_N_ACTIONS ? (int)action[k][i] : 0;
                const int64_t bytes = pk_bytes_per_group(a, P.G);
                const bool fits = (base[k][i] >= 0) & ((base[k][i] & 15) == 0) & (base[k][i] <= P.codes_bytes - bytes * P.R_u);
                kind[k][i] = fits ? a : 0;
                const int64_t group = ((int64_t)rb[i] * P.n_chunks + j) * R_u + lrow;
                s[k][i] = P.scale[group];
                offset[k][i] = P.offset[group];
                const uint32_t per = 0x01023480u >> (4 * a) & 15u;     // bytes of an octet
                const int64_t first = kind[k][i] == 0 ? 0 : base[k][i] + lrow * bytes + (a == 5 ? o * 8u / 5u : o * per);
                v[k][i] = 0;
                if constexpr (WINDOW) {                     // eight bytes within the stream
                    const int64_t from = first < P.codes_bytes - 8 ? first : P.codes_bytes - 8;
                    uint64_t eight;
                    __builtin_memcpy(&eight, P.codes + from, 8);
                    v[k][i] = eight >> (uint32_t)(8 * (first - from));
                } else {
                    for (int b = 0; b < 8; ++b)
                        if (first + b < P.codes_bytes) v[k][i] |= (uint64_t)P.codes[first + b] << (8 * b);
                }
                mask[k][i] = 0;
                if (P.mask != nullptr) mask[k][i] = P.mask[(int64_t)row[i] * P.mask_ld + (col >> 3)];
                kept[k][i][0] = kept[k][i][1] = make_uint4(0u, 0u, 0u, 0u);
                if (kind[k][i] == 0) {
                    const int64_t at = (int64_t)row[i] * P.ld + col;
                    if (P.w_f32 != 0) {
                        kept[k][i][0] = reinterpret_cast<const uint4*>(static_cast<const float*>(P.W) + at)[0];
                        kept[k][i][1] = reinterpret_cast<const uint4*>(static_cast<const float*>(P.W) + at)[1];
                    } else {
                        kept[k][i][0] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(P.W) + at);
                    }
                }
            }
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            float slope;
            const float y = activation<true>(act, bf16_bits_to_f32(g[i]), slope), x = row0 + 64 * i + lane < n_rows ? bf16_bits_to_f32(h[i]) : 0.0f;
            const float d[2] = {x * bf16_bits_to_f32(u[i]) * slope, x * y};
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const PackArgs& P = k == 0 ? gate : up;
                const int a = kind[k][i], b = a == 1 ? 8 : (a == 2 ? 4 : (a == 3 ? 3 : (a == 6 ? 1 : 2)));
                uint32_t lo = (uint32_t)v[k][i];
                const uint32_t hi = a == 1 ? (uint32_t)(v[k][i] >> 32) : 0u;
                if (a == 5) lo = (trit_fields(lo & 0xffu) | trit_fields(lo >> 8 & 0xffu) << 10 | trit_fields(lo >> 16 & 0xffu) << 20) >> (2 * (o * 8u % 5u));
                const float step = a == 6 ? 2.0f : 1.0f, from = a >= 5 ? -1.0f : 0.0f, off = a >= 5 ? 0.0f : offset[k][i];      // code q stands for (step q + from) s + off
                const uint32_t as_is[8] = {kept[k][i][0].x, kept[k][i][0].y, kept[k][i][0].z, kept[k][i][0].w, kept[k][i][1].x, kept[k][i][1].y, kept[k][i][1].z, kept[k][i][1].w};
#pragma unroll
                for (int m = 0; m < 8; ++m) {
                    const float q = (float)__builtin_amdgcn_ubfe(a == 1 && m >= 4 ? hi : lo, (uint32_t)(b * m) & 31u, (uint32_t)b);
                    const uint32_t w16 = (m & 1) != 0 ? as_is[m >> 1] & 0xffff0000u : as_is[m >> 1] << 16;
                    const float coded = (mask[k][i] >> m & 1u) != 0u ? 0.0f : fmaf(fmaf(step, q, from), s[k][i], off), w = __uint_as_float(P.w_f32 != 0 ? as_is[m] : w16);
                    sum[m] = fma((double)d[k], (double)(a == 0 ? w : coded), sum[m]);
                }
            }
        }
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1)
#pragma unroll
        for (int m = 0; m < 8; ++m) sum[m] += __shfl_xor(sum[m], d, 64);
}
__device__ __forceinline__ void dx_again(const PackArgs& gate, const PackArgs& up, int act, const AgainArgs& A, int64_t t, int64_t col, int lane, double (&sum)[8]) {
    if (gate.codes_bytes >= 8 && up.codes_bytes >= 8) dx_again_by<2, true>(gate, up, act, A, t, col, lane, sum);
    else dx_again_by<1, false>(gate, up, act, A, t, col, lane, sum);
}

// H, G and U of a pair's tile: a wavefront has MF x 2 fragments, 2 p and 2 p + 1 along the rows are the gate's and the up's of the same 32 rows.  What is written
// goes through LDS (`out`), one after the other: a lane has four rows of a token, and 8 bytes of each of 32 tokens are written at a third of the rate of whole lines.
template <int MF, int THREADS>
__device__ __forceinline__ void pair_tile(const GemmArgs& Q, f32x16 (&acc)[MF][2], uint16_t* const out, int64_t c0, int64_t t0, int wm, int wn, int tid) {
    constexpr int ROWS = MF * 32, LD = ROWS + 8, WM = MF * 32, TOKENS = THREADS / 2;       // of a token in LDS; of a tile
    const int64_t rows = Q.gate.rows;
    const int lane = tid & 63, sub = lane & 31, hh = lane >> 5;
    // Powers come off; what is then not finite, or lies too low, is noted.  A fragment's powers are loaded while the one before it is gone through.
    float by_token[2];
    float4 next[4];
    auto load_powers = [&](int f) {
#pragma unroll
        for (int g = 0; g < 4; ++g) next[g] = *reinterpret_cast<const float4*>(Q.by_row + c0 + wm * WM + f * 32 + g * 8 + hh * 4);
    };
    load_powers(0);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const int64_t t = t0 + wn * 64 + n * 32 + sub;
        by_token[n] = Q.by_token[t < Q.T ? t : Q.T - 1];
    }
    uint32_t bad = 0;
#pragma unroll
    for (int f = 0; f < MF; ++f) {
        float by[16];
#pragma unroll
        for (int g = 0; g < 4; ++g) by[g * 4] = next[g].x, by[g * 4 + 1] = next[g].y, by[g * 4 + 2] = next[g].z, by[g * 4 + 3] = next[g].w;
        if (f + 1 < MF) load_powers(f + 1);
        asm volatile("" ::: "memory");                      // no others ahead: there are no registers for them
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            uint32_t most = 0;                              // of the magnitudes' bits
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float v = acc[f][n][i];
                acc[f][n][i] = fabsf(v) < loss_in(by_token[n]) + loss_in(by[i]) ? __builtin_nanf("") : ldexpf(v, exponent_of(by_token[n]) + exponent_of(by[i]));
                const uint32_t bits = __float_as_uint(acc[f][n][i]) & 0x7fffffffu;
                most = bits > most ? bits : most;
            }
            bad |= most >= 0x7f800000u ? 1u << (f * 2 + n) : 0u;
        }
    }
    // Weight by weight, a fragment after the other; the code for it once.
    const bool stored[2] = {t0 + wn * 64 + sub < Q.T, t0 + wn * 64 + 32 + sub < Q.T};
    uint32_t todo = 0;
#pragma unroll
    for (int k = 0; k < 2 * MF; ++k) todo |= __any((bad >> k & 1u) != 0u && stored[k & 1] && ((c0 + wm * WM + (k >> 1) * 32) >> 6) * 32 + hh * 4 < rows) ? 1u << k : 0u;
#pragma unroll 1
    for (; todo != 0; todo &= todo - 1) {
        const int which = __builtin_ctz(todo), f = which >> 1, n = which & 1;
        float v[16];
#pragma unroll
        for (int k = 0; k < 2 * MF; ++k)
            if (k == which) {
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = acc[k >> 1][k & 1][i];
            }
        const int64_t first = ((c0 + wm * WM + f * 32) >> 6) * 32 + hh * 4, t = t0 + wn * 64 + n * 32 + sub;
        const GemmArgs& A = argument_in_place<GemmArgs>();
#pragma unroll 1
        for (int i = 0; i < 16; ++i) {
            const int64_t row = first + (i >> 2) * 8 + (i & 3);
            float x = 0.0f;
#pragma unroll
            for (int k = 0; k < 16; ++k) x = i == k ? v[k] : x;
            if (!isfinite(x) && row < rows && t < Q.T) x = (float)pk_slow_dot((f & 1) == 0 ? A.gate : A.pair.up, row, A.raw + t * A.ld_raw);
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = i == k ? x : v[k];
        }
#pragma unroll
        for (int k = 0; k < 2 * MF; ++k)
            if (k == which) {
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[k >> 1][k & 1][i] = v[i];
            }
    }
    auto lay = [&](auto value) {
        __syncthreads();                                    // everybody is done with what lies there
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int p = 0; p < MF / 2; ++p)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    uint32_t v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = f32_to_bf16_bits(value(acc[2 * p][n][g * 4 + i], acc[2 * p + 1][n][g * 4 + i]));
                    *reinterpret_cast<uint2*>(out + (wn * 64 + n * 32 + sub) * LD + wm * (WM / 2) + p * 32 + g * 8 + hh * 4) = make_uint2(v[0] | v[1] << 16, v[2] | v[3] << 16);
                }
        __syncthreads();
    };
    auto write = [&](void* to_, int64_t ld) {
        uint16_t* __restrict__ const to = static_cast<uint16_t*>(to_);
        const bool whole = (ld & 7) == 0 && (reinterpret_cast<uintptr_t>(to) & 15) == 0;
#pragma unroll 4
        for (int i = tid; i < TOKENS * (ROWS / 8); i += THREADS) {
            const int n = i / (ROWS / 8), r = (i - n * (ROWS / 8)) * 8;
            const int64_t t = t0 + n, row = (c0 >> 1) + r;
            if (t >= Q.T || row >= rows) continue;          // rows come in eights
            const uint4 v = *reinterpret_cast<const uint4*>(out + n * LD + r);
            uint16_t* __restrict__ const o = to + t * ld + row;
            if (whole) {
                *reinterpret_cast<uint4*>(o) = v;
            } else {
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int m = 0; m < 8; ++m) o[m] = (uint16_t)(w[m >> 1] >> (16 * (m & 1)));
            }
        }
    };
    if (Q.pair.G != nullptr) {
        lay([](float x, float) { return x; });
        write(Q.pair.G, Q.pair.ld_save);
        lay([](float, float y) { return y; });
        write(Q.pair.U, Q.pair.ld_save);
    }
    lay([&](float x, float y) {
        float none;
        return activation<false>(Q.pair.act, x, none) * y;
    });
    write(Q.dX, Q.ldx);
}

template <int MF, bool HALF = false, bool PAIR = false>    // fragments of a wavefront along the columns; factors in half precision
__global__ __launch_bounds__(GM_THREADS) void dx_gemm_kernel(const GemmArgs Q) {
    constexpr int GM_M = MF * 64, WM = MF * 32, LOADS = (GM_M + GM_N) / 32;
    __shared__ uint4 tile[GM_BUFFERS][(GM_M + GM_N) * 8];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, sub = lane & 31, hh = lane >> 5;
    const int wm = wave & 1, wn = wave >> 1;
    // Consecutive workgroups land on the eight XCDs in turn; each XCD gets a run of tiles, four columns of tiles wide, so that it shares
    // both factors: a run of whole rows of tiles would read all of wt into every XCD's L2.
    const uint32_t n_tiles = gridDim.x, per = n_tiles >> 3;
    const uint32_t id = blockIdx.x < per * 8 ? (blockIdx.x & 7) * per + (blockIdx.x >> 3) : blockIdx.x;
    const uint32_t split = id / (uint32_t)Q.tiles, in = id - split * (uint32_t)Q.tiles, tall = (uint32_t)Q.tiles / Q.col_blocks;
    const uint32_t band = in / (4 * tall), inside = in - band * (4 * tall), width = Q.col_blocks - band * 4 < 4 ? Q.col_blocks - band * 4 : 4;
    const uint32_t tb = inside / width;
    const int64_t c0 = (int64_t)(band * 4 + inside - tb * width) * GM_M, t0 = (int64_t)tb * GM_N;
    const int32_t first = (int32_t)split * Q.each, steps = Q.K / GM_K - first;

    // A lane's share of a tile: slot (lane & 7) of rows 8 wave + lane / 8, 32 rows further on each time; slot p of row r holds the
    // sixteen bytes of slot p ^ (r / 2 & 7).
    const int lr = wave * 8 + (lane >> 3), slot = (lane & 7) ^ ((lr >> 1) & 7);
    const uint16_t* const am = Q.wt + (c0 + lr) * Q.K + first * GM_K + slot * 8;
    const uint16_t* bn[GM_N / 32];
#pragma unroll
    for (int i = 0; i < GM_N / 32; ++i) {
        const int64_t t = t0 + i * 32 + lr;
        bn[i] = Q.dY + (t < Q.T ? t : Q.T - 1) * Q.ldy + first * GM_K + slot * 8;
    }
    const uint32_t lds = lds_address(tile);
    auto load_a = [&](int i, int32_t k, int buf) { lds_load16(lds + (buf * (GM_M + GM_N) * 8 + i * 256 + wave * 64) * 16, am + (int64_t)i * 32 * Q.K + k * GM_K); };
    auto load_b = [&](int i, int32_t k, int buf) { lds_load16(lds + (buf * (GM_M + GM_N) * 8 + GM_M * 8 + i * 256 + wave * 64) * 16, bn[i] + k * GM_K); };
    // Operands of step s (16 of the sum): octet 2 s + hh of a row.
    const uint32_t arow = (wm * WM + sub) * 128, brow = GM_M * 128 + (wn * 64 + sub) * 128;
    auto read_one = [&](int buf, int s, int i, bf16x8 (&a)[MF], bf16x8 (&b)[2]) {
        const char* const at = reinterpret_cast<const char*>(tile[buf]);
        const uint32_t o = (uint32_t)((2 * s + hh) ^ ((sub >> 1) & 7)) * 16;
        if (i < 2) b[i] = as_bf16x8(*reinterpret_cast<const uint4*>(at + brow + i * 32 * 128 + o));
        else a[i - 2] = as_bf16x8(*reinterpret_cast<const uint4*>(at + arow + (i - 2) * 32 * 128 + o));
    };

    const int32_t n_k = steps < Q.each ? steps : Q.each;
    f32x16 acc[MF][2] = {};
    if (n_k > 0) {
#pragma unroll
        for (int i = 0; i < GM_M / 32; ++i) load_a(i, 0, 0);
#pragma unroll
        for (int i = 0; i < GM_N / 32; ++i) load_b(i, 0, 0);
        const int32_t k1 = n_k > 1 ? 1 : 0;
#pragma unroll
        for (int i = 0; i < GM_M / 32; ++i) load_a(i, k1, 1);
#pragma unroll
        for (int i = 0; i < GM_N / 32; ++i) load_b(i, k1, 1);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
        __syncthreads();
        bf16x8 a[2][MF], b[2][2];
#pragma unroll
        for (int i = 0; i < MF + 2; ++i) read_one(0, 0, i, a[0], b[0]);
        int buf = 0;
        for (int32_t k = 0; k < n_k; ++k) {
            const int next = buf == 2 ? 0 : buf + 1, then = next == 2 ? 0 : next + 1;
            const int32_t k2 = k + 2 < n_k ? k + 2 : n_k - 1;       // past the end: again the last, into a buffer that nobody reads
            // Behind every matrix instruction one or two operands of the next step are read, and in the first three steps a load is
            // asked for: put ahead of the instructions they would leave the matrix unit idle for half of the time.
            constexpr int EACH = (LOADS + 2) / 3, MM = MF * 2, READS = (MF + 2 + MM - 2) / (MM - 1);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
#pragma unroll
                for (int i = 0; i < MM; ++i) {
                    if constexpr (HALF)
                        acc[i >> 1][i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a[s & 1][i >> 1]), __builtin_bit_cast(f16x8, b[s & 1][i & 1]), acc[i >> 1][i & 1], 0, 0, 0);
                    else
                        acc[i >> 1][i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[s & 1][i >> 1], b[s & 1][i & 1], acc[i >> 1][i & 1], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    if (s == 3 && i == 0) {
                        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LOADS) : "memory");       // the next buffer's loads are done, this one's reads too
                        __builtin_amdgcn_s_barrier();
                        asm volatile("" ::: "memory");
                    }
#pragma unroll
                    for (int r = i * READS; r < (i + 1) * READS && r < MF + 2; ++r) read_one(s < 3 ? buf : next, s < 3 ? s + 1 : 0, r, a[(s + 1) & 1], b[(s + 1) & 1]);
                    const int j = s * EACH + i;
                    if (s < 3 && i < EACH && j < LOADS) {
                        if (j < GM_M / 32) load_a(j, k2, then);
                        else load_b(j - GM_M / 32, k2, then);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            buf = next;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }

    if constexpr (PAIR) return pair_tile<MF, GM_THREADS>(Q, acc, reinterpret_cast<uint16_t*>(tile), c0, t0, wm, wn, tid);
    if constexpr (HALF) {
        // a tile's octets by lanes
        const int64_t mine = (c0 >> 3) + (lane < GM_M / 8 ? lane : 0), last = (Q.cols >> 3) - 1;
        const float octet_power = Q.by_octet[mine < last ? mine : last];
        const int octet_lost = Q.lost_octet[mine < last ? mine : last];
        auto power_of = [&](int k) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(octet_power), k)); };
        auto below = [&](float by_token, int k) { return lost_below(by_token, power_of(k), __builtin_amdgcn_readlane(octet_lost, k)); };
        const int octet0 = wm * (WM / 8);
        uint32_t todo = 0;                                  // fragments with something that lies too low; of a part of the sum the join says so
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int64_t t = t0 + wn * 64 + n * 32 + sub;
            const float by_token = Q.by_token[t < Q.T ? t : Q.T - 1];
#pragma unroll
            for (int f = 0; f < MF; ++f) {
                bool bad = false;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int64_t c = c0 + wm * WM + f * 32 + g * 8;
                    const float low = below(by_token, octet0 + f * 4 + g);
                    const int by = exponent_of(by_token) + exponent_of(power_of(octet0 + f * 4 + g));
                    float least = fabsf(acc[f][n][g * 4]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        least = fminf(least, fabsf(acc[f][n][g * 4 + i]));
                        acc[f][n][g * 4 + i] = ldexpf(acc[f][n][g * 4 + i], by);
                    }
                    bad |= least < low && c < Q.cols;
                }
                todo |= __any(bad && t < Q.T) ? 1u << (f * 2 + n) : 0u;
            }
        }
        if (Q.part != nullptr) todo = 0;
#pragma unroll 1
        for (; todo != 0; todo &= todo - 1) {
            const int which = __builtin_ctz(todo), f = which >> 1, n = which & 1;
            float v[16];
#pragma unroll
            for (int k = 0; k < 2 * MF; ++k)
                if (k == which) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = acc[k >> 1][k & 1][i];
                }
            const int64_t t = t0 + wn * 64 + n * 32 + sub;
            const float by_token = Q.by_token[t < Q.T ? t : Q.T - 1];
            const GemmArgs& A = argument_in_place<GemmArgs>();
#pragma unroll 1
            for (int g = 0; g < 4; ++g) {
                const int64_t c = c0 + wm * WM + f * 32 + g * 8;
                if (c >= Q.cols) break;
                const float low = below(by_token, octet0 + f * 4 + g);
                const int by = exponent_of(by_token) + exponent_of(power_of(octet0 + f * 4 + g));
                const uint32_t there = (has_codes(power_of(octet0 + f * 4 + g)) || A.lost_octet[c >> 3] != 0 ? 0xffu : A.there_octet[c >> 3]) >> (hh * 4);
                float x[4];
                bool again[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = g == 0 ? v[i] : (g == 1 ? v[4 + i] : (g == 2 ? v[8 + i] : v[12 + i]));
                    again[i] = fabsf(x[i]) < ldexpf(low, by) && t < Q.T && (there >> i & 1u) != 0u;
                }
                const uint64_t lanes = __ballot(again[0] || again[1] || again[2] || again[3]);
#pragma unroll 1
                for (uint32_t left = (uint32_t)lanes | (uint32_t)(lanes >> 32); left != 0; left &= left - 1) {
                    const int token = __builtin_ctz(left);
                    double sum[8];
                    dx_again(A.gate, A.pair.up, A.pair.act, A.again, t0 + wn * 64 + n * 32 + token, c, lane, sum);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (sub == token && again[i]) x[i] = (float)(hh != 0 ? sum[4 + i] : sum[i]);
                }
#pragma unroll
                for (int k = 0; k < 16; ++k) v[k] = g == k >> 2 ? x[k & 3] : v[k];
            }
#pragma unroll
            for (int k = 0; k < 2 * MF; ++k)
                if (k == which) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[k >> 1][k & 1][i] = v[i];
                }
        }
    }
    if (Q.part != nullptr) {
        float* const to = Q.part + (int64_t)split * Q.T * Q.cols;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int64_t t = t0 + wn * 64 + n * 32 + sub;
            if (t >= Q.T) continue;
#pragma unroll
            for (int f = 0; f < MF; ++f)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int64_t c = c0 + wm * WM + f * 32 + g * 8 + hh * 4;
                    if (c < Q.cols) *reinterpret_cast<float4*>(to + t * Q.cols + c) = make_float4(acc[f][n][g * 4], acc[f][n][g * 4 + 1], acc[f][n][g * 4 + 2], acc[f][n][g * 4 + 3]);
                }
        }
        return;
    }
    if (Q.dh != nullptr)
        add_adapters<uint16_t, MF>(Q.A, Q.dh, false, t0 + wn * 64, Q.T, lane, [&](int32_t k, int f) {
            const int64_t c = c0 + wm * WM + f * 32 + sub;
            return Q.at + ((int64_t)k * Q.cols + (c < Q.cols ? c : Q.cols - 1)) * Q.A.max_rank;
        }, acc);

    const bool whole = (Q.ldx & 3) == 0 && (reinterpret_cast<uintptr_t>(Q.dX) & 7) == 0;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const int64_t t = t0 + wn * 64 + n * 32 + sub;
        if (t >= Q.T) continue;
#pragma unroll
        for (int f = 0; f < MF; ++f)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int64_t c = c0 + wm * WM + f * 32 + g * 8 + hh * 4;
                if (c >= Q.cols) continue;                 // columns come in eights
                uint16_t* __restrict__ const o = Q.dX + t * Q.ldx + c;
                uint32_t v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = f32_to_bf16_bits(acc[f][n][g * 4 + i]);
                if (whole) {
                    *reinterpret_cast<uint2*>(o) = make_uint2(v[0] | v[1] << 16, v[2] | v[3] << 16);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[i] = (uint16_t)v[i];
                }
            }
    }
}

#endif  // __HIPCC__

}  // namespace windq
