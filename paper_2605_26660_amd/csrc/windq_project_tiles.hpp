// windq_project for many tokens: tiles of 256 rows x 128 tokens.
//
// Bound by the matrix instructions once a tile's codes are unpacked often enough: 2 T rows cols operations against some 1.2 vector
// instructions per weight and 64 tokens.  Eight wavefronts, four along the rows by two along the tokens, have 64 x 64 results
// each as 2 x 2 fragments of 32x32x16 instructions, two wavefronts per SIMD so that one's unpacking runs under the other's matrix
// instructions.  Weights enter LDS packed: a lane holds one row of a fragment, and which columns its half of the wavefront takes is free as
// long as X's operand does the same, so it takes half a k-block's columns in a row, whose codes are up to 64 contiguous bytes.
//   The two wavefronts of a SIMD do not add up at the same time: one does behind its matrix instructions, the other ahead of its next ones.
//   X and the codes go to LDS by direct loads, one k-block ahead (the next one's load while this one's are used): 128 tokens' octets, and
// for each pair of wavefronts their 64 rows' fields, up to 128 bytes a row.  No register waits for them.  A token's sixteen
// 16-byte slots are exchanged by the token's low bits, so that 32 lanes reading 32 tokens' same slot meet all banks.
//   A k-block's sum over f x is scaled by its group's scale and added to the total in registers: 64 multiply-adds beside
// 32 instructions of 16 K operations.  beta sum x for all k-blocks is a product of its own at the end, with K = k-blocks: both factors as three
// bfloat16 terms, six products in eight of an instruction's sixteen k, so one instruction does two k-blocks.
//   Trits and 3-bit codes are laid out as 2- and 4-bit fields before (by the kernel that sums x): a row of them is visited by
// T / 128 workgroups, and taking trits apart costs more than everything else in the loop.
//   2000 tokens through 4096 x 11008 at 2 bits: 231 us (780 TFLOP/s) + 20 for laying out, 4096 through 13824 x 5120 with 4 adapters of 64 ranks 705 us
// (820 TFLOP/s) + 62; both traced once the card's clock has settled, 251 to 280 and 730 to 920 in the first 10 ms under load.  27560 vector instructions a
// wavefront, 2944 matrix instructions among them: neither unit is full, waits are 46 % of the wavefronts' time.
#pragma once

#include "windq_pair.hpp"

namespace windq {

constexpr int PT_ROWS = 256, PT_TOKENS = 128, PT_THREADS = 512;
constexpr int PT_STRIP = 64;                               // rows of a unit that one workgroup lays out
constexpr int PT_SUMS = 16;                                // tokens whose sums over a k-block one workgroup forms

// Where a unit's fields begin (48 bits of address), how many bits they have (8) and what they are (kind, top byte): 0 skip, 1: 8 bits,
// 2: 4 bits, 4: 2 bits, 5: trits as 2 bits, 6: 1 bit.
typedef unsigned long long UnitWord;
struct KbWord {
    UnitWord fields;           // of the unit's first row in this k-block
    const float* alpha;        // of the unit's first row
};

struct TileArgs {
    PackArgs P;
    const uint16_t* X;         // bfloat16, or the first of three planes
    int64_t ldx, plane;
    const void* raw;
    int64_t ld_raw;
    int64_t T;
    void* Y;
    int64_t ldy;
    const float* h;            // or null: no adapters
    AdapterArgs A;
    uint8_t* fields;           // [U][k-blocks of a chunk][R_u] fields of the units that are laid out anew
    int64_t unit_fields;       // bytes of a unit's
    KbWord* unit;              // [row blocks of units][k-blocks]
    uint4* xs;                 // [k-blocks][T] sum of x as terms
    uint4* beta;               // [k-blocks][rows] beta as terms
    float* alpha;              // [chunks][rows] scales (1 where a unit is skipped)
    int32_t n_kb;              // k-blocks
    uint32_t row_blocks;
    PairArgs pair;             // and what the up matrix has of its own
    KbWord* unit_up;
    uint4* beta_up;
};

// Whether a chunk is one k-block: its rows lie one behind the other in the code stream.  Otherwise every unit is laid out anew, k-block by
// k-block.
__host__ __device__ inline bool tile_natural(int32_t G, int S) { return G == 16 * S; }

// Columns of a k-block / 16, or 0 where the tiles do not fit the shape.
inline int tile_steps(const PackArgs& P) {
    if (P.rows % 8 != 0 || P.rows < PT_STRIP || (P.R_u != P.rows && P.R_u % PT_STRIP != 0)) return 0;
    if (P.G % 128 == 0) return 8;
    if (P.G % 96 == 0) return 6;
    if (P.G % 64 == 0) return 4;
    return 0;
}

#ifdef __HIPCC__

// Workgroups [0, strips): fields of trits and 3-bit codes, every unit's word, and beta of its rows.  The others: sums of x over k-blocks.
template <typename XT, int S>
__global__ __launch_bounds__(256) void tiles_prepare_kernel(const TileArgs Q, const int64_t strips, const int64_t first_block) {
    __shared__ uint16_t trits_of[256];
    const PackArgs& P = Q.P;
    const int32_t per_chunk = P.G / (16 * S);
    const int64_t block = first_block + blockIdx.x;
    if (block >= strips) {
        // sixteen lanes a token, an octet each
        const int64_t first = (block - strips) * PT_SUMS;
        int32_t kb = (int32_t)(first / Q.T);
        int64_t t = first - (int64_t)kb * Q.T + (threadIdx.x >> 4);
        if (t >= Q.T) {                                     // there are more tokens than a workgroup sums up
            t -= Q.T;
            ++kb;
        }
        if (kb >= Q.n_kb) return;
        const int o = threadIdx.x & 15;
        float sum = 0.0f;
        if (o < 2 * S) {
            float v[8];
            load8(static_cast<const XT*>(Q.raw) + t * Q.ld_raw + (int64_t)kb * (16 * S) + o * 8, v);
            sum = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        }
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 16);
        if (o != 0) return;
        uint32_t hi, mid, lo;
        split3(sum, hi, mid, lo);
        Q.xs[(int64_t)kb * Q.T + t] = make_uint4(hi | mid << 16, hi | lo << 16, hi | mid << 16, 0u);
        return;
    }
    const int64_t per_unit = (P.R_u + PT_STRIP - 1) / PT_STRIP;
    const int64_t u = block / per_unit, strip = block - u * per_unit;
    int64_t base;
    const int a = pk_action(P, u, base);
    const bool lay = a == 3 || a == 5 || (a != 0 && !tile_natural(P.G, S));
    uint8_t* __restrict__ const to = Q.fields + u * Q.unit_fields;
    const int64_t rb = u / P.n_chunks, j = u - rb * P.n_chunks;
    {
        const int64_t lrow = strip * PT_STRIP + (threadIdx.x & 63);
        if (lrow < P.R_u) {
            float alpha, beta;
            pk_affine(a == 3 ? 2 : a, P.scale[u * P.R_u + lrow], P.offset[u * P.R_u + lrow], sizeof(XT) == 4, alpha, beta);
            uint32_t hi, mid, lo;
            split3(beta, hi, mid, lo);
            if (threadIdx.x < 64) Q.alpha[j * P.rows + rb * P.R_u + lrow] = alpha;
            for (int32_t c = threadIdx.x >> 6; c < per_chunk; c += 4)
                Q.beta[(j * per_chunk + c) * P.rows + rb * P.R_u + lrow] = make_uint4(hi | hi << 16, mid | hi << 16, lo | mid << 16, 0u);
        }
    }
    if (strip == 0 && threadIdx.x == 0) {
        const UnitWord at = reinterpret_cast<UnitWord>(lay ? to : P.codes + base);
        const UnitWord bits = a == 1 ? 8 : (a == 2 || a == 3 ? 4 : (a == 6 ? 1 : 2));
        for (int32_t c = 0; c < per_chunk; ++c) {
            const UnitWord first = (at + (UnitWord)c * P.R_u * (2 * S * bits)) & 0xffffffffffffull;
            Q.unit[rb * Q.n_kb + j * per_chunk + c] = {a == 0 ? 0ull : first | bits << 48 | (UnitWord)(a == 3 ? 2 : a) << 56, Q.alpha + j * P.rows + rb * P.R_u};
        }
    }
    if (!lay) return;
    if (a == 5) {
        trits_of[threadIdx.x] = (uint16_t)trit_fields(threadIdx.x);
        __syncthreads();
    }
    const int32_t O = P.G >> 3;
    const int64_t nb = pk_bytes_per_group(a, P.G);
    const int64_t left = P.R_u - strip * PT_STRIP;
    const int32_t total = (int32_t)(left < PT_STRIP ? left : PT_STRIP) * O;
    for (int32_t i = threadIdx.x; i < total; i += 256) {
        const int32_t r = i / O, o = i - r * O, c = o / (2 * S);
        const int64_t lrow = strip * PT_STRIP + r;
        const int64_t at = (c * P.R_u + lrow) * (2 * S) + (o - c * 2 * S);      // octets before this one
        const uint8_t* __restrict__ const row = P.codes + base + lrow * nb;
        if (a == 5) {
            reinterpret_cast<uint16_t*>(to)[at] = (uint16_t)octet_trits(row, o, trits_of);
        } else if (a == 3) {
            const uint8_t* p = row + o * 3;
            const uint32_t v = (uint32_t)p[0] | (uint32_t)p[1] << 8 | (uint32_t)p[2] << 16;
            uint32_t w = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) w |= ((v >> (3 * k)) & 7u) << (4 * k);
            reinterpret_cast<uint32_t*>(to)[at] = w;
        } else {
            const int b = a == 1 ? 8 : (a == 2 ? 4 : (a == 4 ? 2 : 1));
            for (int k = 0; k < b; ++k) to[at * b + k] = row[o * b + k];
        }
    }
}

// Masks and leading ones in registers: an and-or takes no constant of its own.
struct TileBits {
    uint32_t mask4 = 0x00780078u, one4 = 0x41804180u, mask2 = 0x00600060u, one2 = 0x40804080u, mask1 = 0x80008000u, one1 = 0x3f803f80u;
    __device__ __forceinline__ TileBits() { asm volatile("" : "+s"(mask4), "+v"(one4), "+s"(mask2), "+v"(one2), "+s"(mask1), "+v"(one1)); }
};

// Octet s of a lane's half row of fields in LDS.
template <int KIND>
struct TileFields {
    uint32_t raw[KIND == 1 ? 16 : (KIND == 2 ? 8 : (KIND == 4 ? 4 : 2))];
    template <int S>
    __device__ __forceinline__ void read(const char* p) {
        constexpr int bytes = S * (KIND == 1 ? 8 : (KIND == 2 ? 4 : (KIND == 4 ? 2 : 1)));
        if constexpr (bytes % 16 == 0) {
#pragma unroll
            for (int i = 0; i < bytes / 16; ++i) {
                const uint4 v = *reinterpret_cast<const uint4*>(p + 16 * i);
                raw[4 * i] = v.x; raw[4 * i + 1] = v.y; raw[4 * i + 2] = v.z; raw[4 * i + 3] = v.w;
            }
        } else if constexpr (bytes % 4 == 0) {
#pragma unroll
            for (int i = 0; i < bytes / 4; ++i) raw[i] = *reinterpret_cast<const uint32_t*>(p + 4 * i);
        } else {                                            // six octets of one bit: rows start on two bytes
            const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
            raw[0] = (uint32_t)q[0] | (uint32_t)q[1] << 16;
            raw[1] = q[2];
        }
        if constexpr (KIND == 6) {
            raw[0] = ~raw[0];
            raw[1] = ~raw[1];
        }
    }
    __device__ __forceinline__ uint4 octet(int s, const TileBits& C) const {
        if constexpr (KIND == 1) return fields8(raw[2 * s], raw[2 * s + 1]);
        else if constexpr (KIND == 2) {
            const uint32_t v = raw[s], e = twice(v, 12, v & 0xffffu), o = twice(v >> 16, 12, v >> 16);
            return make_uint4(((e << 3) & C.mask4) | C.one4, ((e >> 5) & C.mask4) | C.one4, ((o << 3) & C.mask4) | C.one4, ((o >> 5) & C.mask4) | C.one4);
        } else if constexpr (KIND == 4) {
            const uint32_t v = (s & 1) != 0 ? raw[s >> 1] >> 16 : raw[s >> 1] & 0xffffu, t = twice(v, 14, v);
            return make_uint4(((t << 5) & C.mask2) | C.one2, ((t << 1) & C.mask2) | C.one2, ((t >> 3) & C.mask2) | C.one2, ((t >> 7) & C.mask2) | C.one2);
        } else {                                            // of inverted bits: a set one is -1
            const uint32_t v = (raw[s >> 2] >> (8 * (s & 3))) & 0xffu, t = twice(v, 15, v);
            return make_uint4(((t << 15) & C.mask1) | C.one1, ((t << 13) & C.mask1) | C.one1, ((t << 11) & C.mask1) | C.one1, ((t << 9) & C.mask1) | C.one1);
        }
    }
};

// Of a pair (windq_gated) a tile is 128 rows of both: the wavefronts of the lower two strips have the gate's, the others the up's, and those hand their
// results over through LDS at the end.
template <typename YT, int S, bool PAIR = false>
__global__ __launch_bounds__(PT_THREADS) void project_tiles_kernel(const TileArgs Q) {
    constexpr int NP = sizeof(YT) == 4 ? 3 : 1;
    __shared__ uint4 xt[2][PT_TOKENS * 16];
    __shared__ uint4 ct[2][4][512];                        // fields of 64 rows
    __shared__ float st[2][PT_ROWS];
    __shared__ uint4 ring[4][8];                           // units' words, k-block by k-block
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, sub = lane & 31, hh = lane >> 5;
    const int matrix = PAIR ? (wave >> 1) & 1 : 0;
    const PackArgs& P = PAIR && matrix == 1 ? Q.pair.up : Q.P;
    const int wr = wave & 3, wt = wave >> 2;                // wavefronts w and w + 4 share a SIMD, and rows
    // Consecutive workgroups land on the eight XCDs in turn; each XCD gets a run of tiles that share tokens.
    const uint32_t n_tiles = gridDim.x, per = n_tiles >> 3;
    const uint32_t tile = blockIdx.x < per * 8 ? (blockIdx.x & 7) * per + (blockIdx.x >> 3) : blockIdx.x;
    const uint32_t tb = tile / Q.row_blocks;
    const int64_t row0 = (int64_t)(tile - tb * Q.row_blocks) * (PAIR ? PT_ROWS / 2 : PT_ROWS), t0 = (int64_t)tb * PT_TOKENS;

    // X: four of a tile's slots a lane; slot p of token n holds the octet of slot p ^ (n & 15)
    const uint16_t* xsrc[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int n = k * 32 + wave * 4 + (lane >> 4), slot = (lane & 15) ^ (n & 15);
        const int s = (slot & 7) < S ? (slot & 7) : 0;
        const int64_t t = t0 + n;
        xsrc[k] = Q.X + (t < Q.T ? t : Q.T - 1) * Q.ldx + ((slot >> 3) * S + s) * 8;
    }
    // rows: a lane's row of each fragment; the wavefront's unit row block
    const int64_t wrow = row0 + (PAIR ? wr & 1 : wr) * 64;
    const int64_t rb = (wrow < P.rows ? wrow : P.rows - 1) / P.R_u;
    int64_t lrow[2];
#pragma unroll
    for (int f = 0; f < 2; ++f) {
        const int64_t row = wrow + f * 32 + sub;
        lrow[f] = (row < P.rows ? row : P.rows - 1) - rb * P.R_u;
    }
    const int64_t lrow0 = ((wrow < P.rows ? wrow : P.rows - 1) - rb * P.R_u) & ~(int64_t)63;      // a wavefront past the last row loads the last ones
    const int64_t rows_left = P.R_u - lrow0;
    const uint32_t lds_xt = lds_address(xt), lds_ct = lds_address(ct), lds_st = lds_address(st), lds_ring = lds_address(ring);
    const int32_t n_kb = Q.n_kb;
    const KbWord* const words = (PAIR && matrix == 1 ? Q.unit_up : Q.unit) + rb * n_kb;
    const uint4* const betas = PAIR && matrix == 1 ? Q.beta_up : Q.beta;
    auto uniform = [](uint32_t x, uint32_t y) {
        return (UnitWord)(uint32_t)__builtin_amdgcn_readfirstlane((int)y) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
    };
    struct Word {
        UnitWord fields, alpha;
    };
    auto word_of = [&](uint4 w) { return Word{uniform(w.x, w.y), uniform(w.z, w.w)}; };
    auto word_now = [&](int32_t kb) { return word_of(reinterpret_cast<const uint4*>(words)[kb < n_kb ? kb : n_kb - 1]); };
    auto load_word = [&](int32_t kb) {
        if (lane < 4) lds_load4(lds_ring + (wr * 8 + (kb & 7)) * 16, reinterpret_cast<const uint32_t*>(words + (kb < n_kb ? kb : n_kb - 1)) + lane);
    };
    // The fields of the wavefront's 64 rows, 2 S bits bytes a row: every other 64 pieces of 16 bytes by each of the two wavefronts that share them;
    // and the rows' scales, by the one that has read the scales there before by then.
    const uint32_t row_at = (uint32_t)(rows_left < 64 ? (lane < rows_left ? lane : (int32_t)rows_left - 1) : lane);
    auto load_codes = [&](Word word, int32_t kb) {
        const int buf = kb & 1;
        if (wt == 1) lds_load4(lds_st + (buf * PT_ROWS + wr * 64) * 4, reinterpret_cast<const float*>(word.alpha) + lrow0 + row_at);
        if (word.fields == 0) return;
        const int32_t bytes = 2 * S * (int32_t)((uint32_t)(word.fields >> 48) & 0xffu), pieces = 4 * bytes;
        const UnitWord base = (word.fields & 0xffffffffffffull) + (UnitWord)(lrow0 * bytes);
        const int32_t most = (rows_left < 64 ? (int32_t)rows_left * bytes >> 4 : pieces) - 1;
        for (int32_t i0 = wt * 64; i0 < pieces; i0 += 128) {
            const int32_t i = i0 + lane < most ? i0 + lane : most;
            lds_load16(lds_ct + ((buf * 4 + wr) * 512 + i0) * 16, reinterpret_cast<const void*>(base + (uint32_t)(i * 16)));
        }
    };
    auto load_piece = [&](int k, int32_t kb, int p, int buf) {
        lds_load16(lds_xt + (buf * (PT_TOKENS * 16) + k * 512 + wave * 64) * 16, xsrc[k] + p * Q.plane + (int64_t)kb * (16 * S));
    };

    f32x16 tot[2][2] = {};
    const TileBits bits;
    const int32_t n_it = n_kb * NP;                         // k-block by k-block, plane by plane
    Word word = word_now(0), next = word_now(1);
    if (wt == 0) load_word(2);
    load_codes(word, 0);
#pragma unroll
    for (int k = 0; k < 4; ++k) load_piece(k, 0, 0, 0);
    f32x16 acc[2][2];
    // A k-block's sums times its groups' scales, added to the total.
    auto fold = [&](int32_t kb) {
        const float* const sc = st[kb & 1] + wr * 64 + 4 * hh;
        float4 a[2][4];
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int g = 0; g < 4; ++g) a[f][g] = *reinterpret_cast<const float4*>(sc + f * 32 + g * 8);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float av[4] = {a[f][g].x, a[f][g].y, a[f][g].z, a[f][g].w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int n = 0; n < 2; ++n) tot[f][n][g * 4 + i] = fmaf(av[i], acc[f][n][g * 4 + i], tot[f][n][g * 4 + i]);
            }
    };
    int32_t kb = 0;
    int plane = 0;
    for (int32_t it = 0; it < n_it; ++it) {
        const int buf = it & 1;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const int kind = (int)(word.fields >> 56);
        const bool last = plane == NP - 1;                  // of the k-block's planes
        if (wt == 1 && plane == 0 && it > 0) {
            fold(kb - 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        // The next iteration's data.  The last one asks for its own again, into places that nobody reads any more: a branch would cost more.
        const int32_t kb_then = last && kb + 1 < n_kb ? kb + 1 : kb;
        const int plane_then = last ? 0 : plane + 1;
        if (last) {
            if (wt == 0) load_word(kb + 3);
            load_codes(next, kb + 1);
        }
        if (plane == 0) {
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
                for (int n = 0; n < 2; ++n) acc[f][n] = f32x16{};
        }
        const uint32_t xb = (uint32_t)buf * sizeof(xt[0]) + (wt * 64 + sub) * 256 + (((hh * 8) ^ (sub & 15)) << 4);
        const char* const cb = reinterpret_cast<const char*>(ct[kb & 1][wr]);
        auto tokens_of = [&](int s, bf16x8 (&b)[2]) {
            const char* const at = reinterpret_cast<const char*>(xt) + (xb ^ (uint32_t)(s << 4));
            b[0] = as_bf16x8(*reinterpret_cast<const uint4*>(at));
            b[1] = as_bf16x8(*reinterpret_cast<const uint4*>(at + 32 * 256));
        };
        auto multiply = [&](const uint4 (&a)[2], const bf16x8 (&b)[2]) {
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
                for (int n = 0; n < 2; ++n) acc[f][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a[f]), b[n], acc[f][n], 0, 0, 0);
        };
        // While one step's four matrix instructions run, the next one's codes are unpacked, six vector instructions behind each, and
        // the tokens of the step DEPTH on are read: LDS takes longer than one step.  The next k-block's X is asked for in between, a
        // piece a step: 64 lanes' 16 bytes keep the way to LDS busy for 16 clocks, and who asks for more at once waits for it.
        auto steps = [&](auto fields, int row_bytes) {
            decltype(fields) v[2];
            auto octet = [&](int f, int s) { return NP == 3 ? centred(v[f].octet(s, bits), pk_centre(kind)) : v[f].octet(s, bits); };
            constexpr int DEPTH = 2;
            bf16x8 b[DEPTH + 1][2];
            uint4 a[2][2];
            v[0].template read<S>(cb + sub * row_bytes + hh * (row_bytes >> 1));
            v[1].template read<S>(cb + (32 + sub) * row_bytes + hh * (row_bytes >> 1));
#pragma unroll
            for (int s = 0; s < DEPTH; ++s) tokens_of(s, b[s]);
            a[0][0] = octet(0, 0);
            a[0][1] = octet(1, 0);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int s = 0; s < S; ++s) {
                if (s < 4) load_piece(s, kb_then, plane_then, buf ^ 1);
                if (s + DEPTH < S) tokens_of(s + DEPTH, b[(s + DEPTH) % (DEPTH + 1)]);
                if (s + 1 < S) {
                    a[(s + 1) & 1][0] = octet(0, s + 1);
                    a[(s + 1) & 1][1] = octet(1, s + 1);
                }
                multiply(a[s & 1], b[s % (DEPTH + 1)]);
                if (s + DEPTH < S) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                if (s + 1 < S) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        if (kind == 6) {
            steps(TileFields<6>(), 2 * S);
        } else if (kind == 4 || kind == 5) {
            steps(TileFields<4>(), 4 * S);
        } else if (kind == 2) {
            steps(TileFields<2>(), 8 * S);
        } else if (kind == 1) {
            steps(TileFields<1>(), 16 * S);
        } else {
            const int64_t c = (int64_t)kb * (16 * S) + hh * (8 * S);
#pragma unroll
            for (int k = 0; k < 4; ++k) load_piece(k, kb_then, plane_then, buf ^ 1);
            const int terms = P.w_f32 != 0 ? 3 - plane : 1;       // of a weight's terms with this plane's: those that count
            for (int term = 0; term < terms; ++term) {
#pragma unroll 2
                for (int s = 0; s < S; ++s) {
                    bf16x8 b[2];
                    tokens_of(s, b);
                    multiply({skip_octet(P, rb * P.R_u + lrow[0], c + s * 8, term), skip_octet(P, rb * P.R_u + lrow[1], c + s * 8, term)}, b);
                }
            }
        }
        if (last) {
            if (wt == 0) fold(kb);
            word = next;
            ++kb;
            next = word_of(ring[wr][(kb + 1) & 7]);         // asked for a k-block ago
            plane = 0;
        } else {
            ++plane;
        }
    }
    if (wt == 1) fold(n_kb - 1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

    // beta sum x, two k-blocks an instruction
    int64_t tok[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        tok[n] = t0 + wt * 64 + n * 32 + sub;
        if (tok[n] >= Q.T) tok[n] = Q.T - 1;
    }
    constexpr int ROUND = 6;                                // pairs of k-blocks whose operands are on their way together
    const uint4 nothing = make_uint4(0u, 0u, 0u, 0u);
    for (int32_t k0 = 0; k0 < n_kb; k0 += 2 * ROUND) {
        uint4 a[ROUND][2], b[ROUND][2];
#pragma unroll
        for (int k = 0; k < ROUND; ++k) {
            const int32_t at = k0 + 2 * k + hh < n_kb ? k0 + 2 * k + hh : n_kb - 1;
#pragma unroll
            for (int f = 0; f < 2; ++f) a[k][f] = betas[at * P.rows + rb * P.R_u + lrow[f]];
#pragma unroll
            for (int n = 0; n < 2; ++n) b[k][n] = Q.xs[at * Q.T + tok[n]];
        }
#pragma unroll
        for (int k = 0; k < ROUND; ++k) {
            const bool in = k0 + 2 * k + hh < n_kb;
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
                for (int n = 0; n < 2; ++n)
                    tot[f][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(in ? a[k][f] : nothing), as_bf16x8(in ? b[k][n] : nothing), tot[f][n], 0, 0, 0);
        }
    }

    // what is not finite so far: weight by weight
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            bool bad = false;
#pragma unroll
            for (int i = 0; i < 16; ++i) bad |= !isfinite(tot[f][n][i]);
            if (__any(bad)) {
                for (int i = 0; i < 16; ++i) {
                    const int64_t row = wrow + f * 32 + (i >> 2) * 8 + hh * 4 + (i & 3), t = t0 + wt * 64 + n * 32 + sub;
                    float v = 0.0f;
#pragma unroll
                    for (int k = 0; k < 16; ++k) v = i == k ? tot[f][n][k] : v;
                    if (!isfinite(v) && row < P.rows && t < Q.T) v = (float)pk_slow_dot(P, row, static_cast<const YT*>(Q.raw) + t * Q.ld_raw);
#pragma unroll
                    for (int k = 0; k < 16; ++k) tot[f][n][k] = i == k ? v : tot[f][n][k];
                }
            }
        }

    if (!PAIR && Q.h != nullptr)
        add_adapters<YT, 2>(Q.A, Q.h, true, t0 + wt * 64, Q.T, lane,
                            [&](int32_t k, int f) { return static_cast<const YT*>(Q.A.b) + ((int64_t)k * P.rows + rb * P.R_u + lrow[f]) * Q.A.max_rank; }, tot);

    auto store = [&](void* to, int64_t ld) {
        YT* __restrict__ const Y = static_cast<YT*>(to);
        const bool whole = (ld & 3) == 0 && (reinterpret_cast<uintptr_t>(Y) & (4 * sizeof(YT) - 1)) == 0;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int64_t t = t0 + wt * 64 + n * 32 + sub;
            if (t >= Q.T) continue;
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int64_t row = wrow + f * 32 + g * 8 + hh * 4;
                    if (row >= P.rows) continue;           // rows come in eights
                    YT* __restrict__ const o = Y + t * ld + row;
                    float v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = tot[f][n][g * 4 + i];
                    if (whole) {
                        if constexpr (sizeof(YT) == 4) *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
                        else *reinterpret_cast<uint2*>(o) = make_uint2(f32_to_bf16_bits(v[0]) | f32_to_bf16_bits(v[1]) << 16, f32_to_bf16_bits(v[2]) | f32_to_bf16_bits(v[3]) << 16);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if constexpr (sizeof(YT) == 4) o[i] = v[i];
                            else o[i] = (uint16_t)f32_to_bf16_bits(v[i]);
                        }
                    }
                }
        }
    };
    if constexpr (PAIR) {
        if (Q.pair.G != nullptr) store(matrix == 1 ? Q.pair.U : Q.pair.G, Q.pair.ld_save);
        float* const over = reinterpret_cast<float*>(xt) + ((wr & 1) * 2 + wt) * 4096 + lane;    // 64 results a lane
        static_assert(sizeof(xt) >= 4 * 4096 * sizeof(float), "the up's results fit");
        __syncthreads();                                    // everybody is done with X
        if (matrix == 1) {
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int i = 0; i < 16; ++i) over[((f * 2 + n) * 16 + i) * 64] = tot[f][n][i];
        }
        __syncthreads();
        if (matrix == 1) return;
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float none;
                    tot[f][n][i] = activation<false>(Q.pair.act, tot[f][n][i], none) * over[((f * 2 + n) * 16 + i) * 64];
                }
    }
    store(Q.Y, Q.ldy);
}

#endif  // __HIPCC__

}  // namespace windq
