// 8-bit tokens (windq_tokens8), a plan's form for serving them (windq_serving_lay), and their products (windq_project8, windq_gated8).
#include <math.h>

#include "windq_eight_tiles.hpp"

namespace windq {

// ------------------------------------------------------------------------------------------------ tokens
// A workgroup a token, its octets (of the padded width) to neighbouring threads, read once where a thread has PER of them at most: they stay in registers
// between the pass for the largest magnitude and the one that rounds.  Magnitudes are compared as bits: a NaN's are above an infinity's, and those above
// every number's.  A k-block's sum is formed by the lanes that have it where they are 4, 8 or 16 together, else by integer additions in LDS, whose order does not matter.
constexpr int TOKENS_SUMS = 4096;                          // k-blocks whose sums fit

struct TokensArgs {
    const void* X;
    int64_t ld, T;
    int8_t* codes;
    float* scale;
    int32_t* sums;
    int32_t G, octets_chunk;   // octets of a chunk with its padding
    int32_t octets_kb;
    int64_t octets, sums_ld;   // of the padded width
    int32_t n_kb;
};

template <typename XT, int PER>                            // 0: any number of octets a thread, read twice
__global__ __launch_bounds__(256) void tokens8_kernel(const TokensArgs Q, const int64_t first) {
    constexpr bool F32 = sizeof(XT) == 4;
    __shared__ uint32_t most[4];
    __shared__ int32_t sums[TOKENS_SUMS];
    const int64_t t = first + blockIdx.x;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const XT* __restrict__ const x = static_cast<const XT*>(Q.X) + t * Q.ld;
    const bool natural = Q.octets_chunk * 8 == Q.G, whole = Q.octets_kb != 12, own_sums = Q.n_kb <= TOKENS_SUMS;
    if (own_sums && !whole) {
        for (int32_t k = threadIdx.x; k < Q.n_kb; k += 256) sums[k] = 0;
        __syncthreads();
    }
    auto load = [&](int64_t o, uint4 (&v)[F32 ? 2 : 1]) {   // zeros past the end and in the padding
        int64_t at = o * 8;
        bool in = o < Q.octets;
        if (!natural) {
            const int64_t j = (int64_t)((uint64_t)o / (uint32_t)Q.octets_chunk);
            const int32_t c = (int32_t)(o - j * Q.octets_chunk) * 8;
            in = in && c < Q.G;
            at = j * Q.G + c;
        }
#pragma unroll
        for (int k = 0; k < (F32 ? 2 : 1); ++k) v[k] = in ? reinterpret_cast<const uint4*>(x + at)[k] : make_uint4(0u, 0u, 0u, 0u);
    };
    auto value = [&](const uint4 (&v)[F32 ? 2 : 1], int i) {
        const uint4 w = v[F32 ? i >> 2 : 0];
        const int k = F32 ? i & 3 : i >> 1;
        const uint32_t b = k == 0 ? w.x : (k == 1 ? w.y : (k == 2 ? w.z : w.w));
        return F32 ? b : ((i & 1) != 0 ? b & 0xffff0000u : b << 16);
    };
    uint32_t m = 0;                                         // of bfloat16 a pair of them
    auto largest = [&](const uint4 (&v)[F32 ? 2 : 1]) {
#pragma unroll
        for (int k = 0; k < (F32 ? 2 : 1); ++k) {
            const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (F32) {
                    const uint32_t b = w[i] & 0x7fffffffu;
                    m = b > m ? b : m;
                } else {
                    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
                    m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m), __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu)));
                }
            }
        }
    };
    uint4 held[PER > 0 ? PER : 1][F32 ? 2 : 1];
    if constexpr (PER > 0) {
#pragma unroll
        for (int k = 0; k < PER; ++k) load(k * 256 + threadIdx.x, held[k]);
#pragma unroll
        for (int k = 0; k < PER; ++k) largest(held[k]);
    } else {
        for (int64_t o = threadIdx.x; o < Q.octets; o += 256) {
            load(o, held[0]);
            largest(held[0]);
        }
    }
    if constexpr (!F32) m = m << 16 > (m & 0xffff0000u) ? m << 16 : m & 0xffff0000u;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        const uint32_t b = (uint32_t)__shfl_xor((int)m, d, 64);
        m = b > m ? b : m;
    }
    if (lane == 0) most[wave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) m = most[w] > m ? most[w] : m;
    const bool finite = m < 0x7f800000u;
    float sigma = __uint_as_float(m) / 127.0f;
    if (sigma < 1.17549435e-38f) sigma = 0.0f;
    const float inverse = finite && sigma > 0.0f ? 1.0f / sigma : 0.0f;
    if (threadIdx.x == 0) Q.scale[t] = finite ? sigma : __uint_as_float(0x7fc00000u);
    uint2* __restrict__ const to = reinterpret_cast<uint2*>(Q.codes + t * Q.octets * 8);
    // x / sigma is at most 127 (1 + 2^-22): no clamp.  1.5 2^23 added, the sum's last bits are the integer, ties to even.
    auto round = [&](int64_t o, const uint4 (&v)[F32 ? 2 : 1]) {
        uint32_t w[2];
        int32_t sum = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float y = __uint_as_float(value(v, h * 4 + i)) * inverse;
                q[i] = __float_as_uint(y + 12582912.0f);
            }
            const uint32_t lo = __builtin_amdgcn_perm(q[1], q[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(q[3], q[2], 0x04000c0cu);
            w[h] = finite ? lo | hi : 0u;
            sum = __builtin_amdgcn_sdot4((int)w[h], 0x01010101, sum, false);
        }
        if (o < Q.octets) to[o] = make_uint2(w[0], w[1]);
        if (!own_sums) return;
        if (whole) {
            for (int d = 1; d < Q.octets_kb; d <<= 1) sum += __shfl_xor(sum, d, 64);
            if (o < Q.octets && (o & (Q.octets_kb - 1)) == 0) Q.sums[t * Q.sums_ld + o / Q.octets_kb] = sum;
        } else if (o < Q.octets && sum != 0) {
            atomicAdd(&sums[(uint32_t)o / (uint32_t)Q.octets_kb], sum);
        }
    };
    if constexpr (PER > 0) {
#pragma unroll
        for (int k = 0; k < PER; ++k) round(k * 256 + threadIdx.x, held[k]);
    } else {
        for (int64_t o0 = 0; o0 < Q.octets; o0 += 256) {    // all lanes: they sum up together
            load(o0 + threadIdx.x, held[0]);
            round(o0 + threadIdx.x, held[0]);
        }
    }
    if (!own_sums) return;
    if (whole) {
        if (threadIdx.x < Q.sums_ld - Q.n_kb) Q.sums[t * Q.sums_ld + Q.n_kb + threadIdx.x] = 0;
        return;
    }
    __syncthreads();
    for (int64_t k = threadIdx.x; k < Q.sums_ld; k += 256) Q.sums[t * Q.sums_ld + k] = k < Q.n_kb ? sums[k] : 0;
}

template <typename XT>
int launch_tokens8(const TokensArgs& Q, hipStream_t st) {
    const int64_t each = tokens_in(Q.octets, 256);
    return launch_pieces(Q.T, 256, [&](int64_t first, dim3 g) {
        if (each <= 1) tokens8_kernel<XT, 1><<<g, dim3(256), 0, st>>>(Q, first);
        else if (each <= 2) tokens8_kernel<XT, 2><<<g, dim3(256), 0, st>>>(Q, first);
        else if (each <= 3) tokens8_kernel<XT, 3><<<g, dim3(256), 0, st>>>(Q, first);
        else if (each <= 4) tokens8_kernel<XT, 4><<<g, dim3(256), 0, st>>>(Q, first);
        else if (each <= 6) tokens8_kernel<XT, 6><<<g, dim3(256), 0, st>>>(Q, first);
        else if (each <= 8) tokens8_kernel<XT, 8><<<g, dim3(256), 0, st>>>(Q, first);
        else tokens8_kernel<XT, 0><<<g, dim3(256), 0, st>>>(Q, first);
    });
}

// Sums of tokens of more k-blocks than fit LDS, a thread a sum, from the codes.
__global__ __launch_bounds__(256) void tokens8_sums_kernel(const TokensArgs Q, const int64_t first) {
    const int64_t i = (first + blockIdx.x) * 256 + threadIdx.x;
    if (i >= Q.T * Q.sums_ld) return;
    const int64_t t = i / Q.sums_ld, k = i - t * Q.sums_ld;
    int32_t sum = 0;
    if (k < Q.n_kb)
        for (int32_t c = 0; c < Q.octets_kb * 8; ++c) sum += Q.codes[t * Q.octets * 8 + k * Q.octets_kb * 8 + c];
    Q.sums[i] = sum;
}

// ------------------------------------------------------------------------------------------------ the plan's form for serving
// A wavefront a row block of a unit and k-block; a lane gathers its 16 columns of every step.  Laid once, bound by nothing in particular.
__device__ __forceinline__ int eight_code(int a, const uint8_t* __restrict__ row, int c) {
    switch (a) {
        case 1: return (int)row[c] - 128;
        case 2: return (row[c >> 1] >> (4 * (c & 1))) & 15;
        case 3: {
            const int bit = 3 * c;
            const uint32_t v = (uint32_t)row[bit >> 3] | ((bit & 7) > 5 ? (uint32_t)row[(bit >> 3) + 1] << 8 : 0u);
            return (int)((v >> (bit & 7)) & 7u);
        }
        case 4: return (row[c >> 2] >> (2 * (c & 3))) & 3;
        case 5: {
            uint32_t v = row[c / 5];
            for (int i = c % 5; i > 0; --i) v /= 3u;
            return (int)(v % 3u);
        }
        default: return (row[c >> 3] >> (c & 7)) & 1;
    }
}

__global__ __launch_bounds__(256) void serving_lay_kernel(const PackArgs P, const EightShape E, const int64_t* __restrict__ image_off, char* __restrict__ image,
                                                          const int64_t bytes, const int64_t first) {
    const int64_t id = (first + blockIdx.x) * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, sub = lane & 31, hh = lane >> 5;
    const int64_t per_unit = E.RB * E.per_chunk;
    const int64_t u = id / per_unit;
    if (u >= E.U) return;
    const int64_t i = (id - u * per_unit) / E.per_chunk;
    const int32_t c = (int32_t)(id - u * per_unit - i * E.per_chunk);
    const int64_t rb = u / E.n_chunks, j = u - rb * E.n_chunks;
    int64_t base;
    const int a = pk_action(P, u, base);
    int kind = eight_kind(a);
    const int64_t block = eight_bytes(kind, E.S, P.w_f32 != 0), need = block * per_unit, at = image_off[u], end = image_off[u + 1];
    if (at < E.header || (at & 255) != 0 || end > bytes || end - at < need || at > bytes - EIGHT_PAST - need) kind = EIGHT_NOTHING;
    const int64_t mine = (rb * E.RB + i) * E.n_kb + j * E.per_chunk + c;
    const int64_t here = at + (i * E.per_chunk + c) * block;
    if (lane == 0) reinterpret_cast<uint32_t*>(image)[mine] = kind == EIGHT_NOTHING ? (uint32_t)kind : (uint32_t)(here >> 8) << 3 | (uint32_t)kind;
    const int64_t lrow = i * EIGHT_ROWS + sub;
    const bool in = lrow < P.R_u;
    const int64_t row = rb * P.R_u + (in ? lrow : 0);
    {
        const float scale = in ? P.scale[u * P.R_u + lrow] : 0.0f, offset = in ? P.offset[u * P.R_u + lrow] : 0.0f;
        float alpha = scale, beta = offset;
        if (a == 1) beta = fmaf(128.0f, scale, offset);
        if (a == 5) beta = -scale;
        if (a == 6) {
            alpha = 2.0f * scale;
            beta = -scale;
        }
        if (kind == 0 || kind == EIGHT_NOTHING) {
            alpha = in && kind == 0 ? 1.0f : 0.0f;
            beta = 0.0f;
        }
        float* const to = reinterpret_cast<float*>(image + E.affine) + mine * 64;
        to[hh * 32 + sub] = hh == 0 ? alpha : beta;
    }
    if (kind == EIGHT_NOTHING) return;
    char* const to = image + here;
    const uint8_t* const codes = P.codes + base + (in ? lrow : 0) * pk_bytes_per_group(a, P.G);
    uint32_t bits = 0;
    for (int s = 0; s < E.S; ++s) {
        const int32_t c0 = (c * E.S + s) * 32 + hh * 16;    // of the chunk's columns
        if (kind == 0) {
            for (int half = 0; half < 2; ++half) {
                const int32_t col = c0 + half * 8;
                const int terms = P.w_f32 != 0 ? 3 : 1;
                for (int term = 0; term < terms; ++term) {
                    const uint4 w = in && col < P.G ? skip_octet(P, row, j * P.G + col, term) : make_uint4(0u, 0u, 0u, 0u);
                    reinterpret_cast<uint4*>(to)[((s * terms + term) * 2 + half) * 64 + lane] = w;
                }
            }
            continue;
        }
        uint32_t v[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] = in && c0 + k < P.G ? (uint32_t)eight_code(a, codes, c0 + k) : 0u;
        // words of a lane's string, each to its piece
        auto put = [&](int k, uint32_t w) {
            const int length = eight_string(kind, E.S), full = length >> 4;
            char* const p = (k >> 2) < full ? to + (k >> 2) * 1024 + lane * 16 : to + full * 1024 + lane * (length & 15);
            reinterpret_cast<uint32_t*>(p)[k & 3] = w;
        };
        uint32_t w[4] = {};
        if (kind == 1) {
#pragma unroll
            for (int k = 0; k < 16; ++k) w[k >> 2] |= (v[k] & 0xffu) << (8 * (k & 3));
            for (int k = 0; k < 4; ++k) put(4 * s + k, w[k]);
        } else if (kind == 2) {
#pragma unroll
            for (int k = 0; k < 16; ++k) w[k >> 3] |= v[k] << (8 * (k & 3) + 4 * ((k >> 2) & 1));
            put(2 * s, w[0]);
            put(2 * s + 1, w[1]);
        } else if (kind == 4) {
#pragma unroll
            for (int k = 0; k < 16; ++k) w[0] |= v[k] << (8 * (k & 3) + 2 * (k >> 2));
            put(s, w[0]);
        } else {
#pragma unroll
            for (int k = 0; k < 16; ++k) bits |= v[k] << (8 * (k & 3) + (k >> 2) + 4 * (s & 1));
            if ((s & 1) != 0 || s + 1 == E.S) {
                put(s >> 1, bits);
                bits = 0;
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------ the product
// Whether the kernel for few tokens is the faster one beyond 32 of them, by rounds of workgroups on 256 CUs: one of its own takes 0.23 us a k-block (of a pair 0.45),
// one of tiles 1.1 (1.25) while there is one, 0.8 (1.0) each where two share a CU.  32 k-blocks, 11008 rows: 128 tokens (three rounds) 26 us, tiles 37; 256 tokens
// (six) 50 and 38; 4096 rows: 512 tokens (four) 34 and 37, 768 (six) 50 and 38; a pair of 11008 rows: 64 tokens (two) 33 and 42, 96 (three) 47 and 44.
inline bool eight_few(int64_t workgroups, int64_t tiles, bool pair) {
    const int64_t rounds = tokens_in(workgroups, 256), by_tiles = tokens_in(tiles, 256);
    return 10 * rounds <= (pair ? (by_tiles == 1 ? 27 : 22 * by_tiles) : (by_tiles == 1 ? 48 : 35 * by_tiles));
}

// A row block and 32 N tokens a workgroup; its wavefronts share the k-blocks (of a pair: half of them the gate's, the others the up's) and
// add up through LDS.  Bound by latency: everything that a k-block needs is asked for at once, and the next one's fields before this one is multiplied.
// Tokens are the M side of the matrix instructions and rows the N side, so that a lane has one row, with one alpha and one beta; beta times the tokens' sums
// is an instruction of its own, whose halves have the sums of a step's halves.  Tokens come through a place of the wavefront's own in LDS, whole lines
// of eight of them at a time: 16 bytes of each of 32 tokens in one load are 32 lines (48 tokens through 11008 x 4096 22 us, 17 so; a pair of them at 16 tokens 19 and 14).
template <typename YT, int S, int N, int WAVES, bool PAIR>
__global__ __launch_bounds__(WAVES * 64) void eight_kernel(const EightArgs Q, const int64_t first) {
    constexpr int EACH = PAIR ? WAVES / 2 : WAVES;
    __shared__ uint4 mem[WAVES][N * 256];                   // a wavefront's tokens, 128 bytes each, and its results later
    float(*const red)[N * 16][64] = reinterpret_cast<float(*)[N * 16][64]>(mem);
    static_assert(sizeof(mem) == WAVES * N * 16 * 64 * sizeof(float), "results fit");
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, sub = lane & 31, hh = lane >> 5;
    const int turn = wave % EACH;
    const EightPlan& P = Q.P[PAIR ? wave / EACH : 0];
    const int64_t id = first + blockIdx.x, tb = id / Q.NB, b = id - tb * Q.NB, t0 = tb * (N * 32);
    const int64_t rb = b / Q.RB, i = b - rb * Q.RB;
    const bool w_f32 = Q.w_f32 != 0;

    // slot p of a token's eight holds the sixteen bytes of slot p ^ (token / 2 & 7)
    const int8_t* x[N * 4];
#pragma unroll
    for (int k = 0; k < N * 4; ++k) {
        const int n = k * 8 + (lane >> 3), slot = (lane & 7) ^ ((n >> 1) & 7);
        x[k] = Q.codes + (t0 + n < Q.T ? t0 + n : Q.T - 1) * Q.width + (slot < 2 * S ? slot : 0) * 16;
    }
    const uint32_t lds = lds_address(mem[wave]);
    const char* const place = reinterpret_cast<const char*>(mem[wave]) + sub * 128;
    const uint32_t* const words = reinterpret_cast<const uint32_t*>(P.image) + b * Q.n_kb;
    const float* const affine = reinterpret_cast<const float*>(P.image + Q.affine) + b * Q.n_kb * 64 + sub;
    f32x16 tot[N] = {};
    for (int32_t from = turn; from < Q.n_kb; from += 64 * EACH) {
        // the words of the wavefront's next 64 k-blocks, a lane each
        const int32_t mine = from + lane * EACH;
        const uint32_t of = mine < Q.n_kb ? eight_word(P, words[mine], S, w_f32) : (uint32_t)EIGHT_NOTHING;
        const int32_t count = (Q.n_kb - from + EACH - 1) / EACH < 64 ? (Q.n_kb - from + EACH - 1) / EACH : 64;
        EightBlock u = eight_block(P, (uint32_t)__builtin_amdgcn_readlane((int)of, 0));
        EightFields<S> raw;
        raw.load(u.kind, u.fields, lane);
        for (int32_t it = 0; it < count; ++it) {
            const int32_t kb = from + it * EACH;
            const int kind = u.kind;
#pragma unroll
            for (int k = 0; k < N * 4; ++k)
                if (t0 + k * 8 < Q.T) lds_load16(lds + k * 1024, x[k] + (int64_t)kb * (32 * S));       // past the last token: whatever lies there, for results that nobody stores
            const float alpha = affine[(int64_t)kb * 64], beta = affine[(int64_t)kb * 64 + 32];
            i32x4 w[S];
            raw.operands(kind, w);
            const EightBlock here = u;
            wait_for_loads();
            u = eight_block(P, (uint32_t)__builtin_amdgcn_readlane((int)of, it + 1 < count ? it + 1 : it));
            raw.load(u.kind, u.fields, lane);
            uint4 xv[S][N];
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int n = 0; n < N; ++n) xv[s][n] = *reinterpret_cast<const uint4*>(place + n * 4096 + (((2 * s + hh) ^ ((sub >> 1) & 7)) << 4));
            if (kind == 0) {
                const int terms = w_f32 ? 3 : 1;
                const uint4* const weights = reinterpret_cast<const uint4*>(here.fields) + lane;
#pragma unroll 1
                for (int term = 0; term < terms; ++term) {
                    uint4 v[S][2];
#pragma unroll
                    for (int s = 0; s < S; ++s)
#pragma unroll
                        for (int half = 0; half < 2; ++half) v[s][half] = weights[((s * terms + term) * 2 + half) * 64];
#pragma unroll
                    for (int s = 0; s < S; ++s)
#pragma unroll
                        for (int n = 0; n < N; ++n) {
                            tot[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(eight_as_bf16(xv[s][n].x, xv[s][n].y), as_bf16x8(v[s][0]), tot[n], 0, 0, 0);
                            tot[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(eight_as_bf16(xv[s][n].z, xv[s][n].w), as_bf16x8(v[s][1]), tot[n], 0, 0, 0);
                        }
                }
                continue;
            }
            i32x16 acc[N];
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int n = 0; n < N; ++n) acc[n] = __builtin_amdgcn_mfma_i32_32x32x32_i8(as_i32x4(xv[s][n]), w[s], s == 0 ? i32x16{} : acc[n], 0, 0, 0);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                int sum = 0;
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    sum = __builtin_amdgcn_sdot4((int)xv[s][n].x, 0x01010101, sum, false);
                    sum = __builtin_amdgcn_sdot4((int)xv[s][n].y, 0x01010101, sum, false);
                    sum = __builtin_amdgcn_sdot4((int)xv[s][n].z, 0x01010101, sum, false);
                    sum = __builtin_amdgcn_sdot4((int)xv[s][n].w, 0x01010101, sum, false);
                }
                tot[n] = __builtin_amdgcn_mfma_f32_32x32x2f32((float)sum, beta, tot[n], 0, 0, 0);
            }
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int k = 0; k < 16; ++k) tot[n][k] = fmaf(alpha, (float)acc[n][k], tot[n][k]);
        }
    }
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int k = 0; k < 16; ++k) red[wave][n * 16 + k][lane] = tot[n][k];
    __syncthreads();
    const int32_t rows_left = Q.R_u - i * EIGHT_ROWS < EIGHT_ROWS ? (int32_t)(Q.R_u - i * EIGHT_ROWS) : EIGHT_ROWS;
    for (int e = threadIdx.x; e < N * 1024; e += WAVES * 64) {
        const int r = e & 31, n = e >> 5;                  // neighbouring lanes: neighbouring rows of a token
        const int64_t t = t0 + n;
        if (r >= rows_left || t >= Q.T) continue;
        const int slot = (n >> 5) * 16 + ((n >> 3) & 3) * 4 + (n & 3), at = ((n >> 2) & 1) * 32 + r;
        float v = 0.0f, up = 0.0f;
#pragma unroll
        for (int w = 0; w < EACH; ++w) v += red[w][slot][at];
        const float scale = Q.scale[t];
        v *= scale;
        if constexpr (PAIR) {
#pragma unroll
            for (int w = EACH; w < WAVES; ++w) up += red[w][slot][at];
            float none;
            v = activation<false>(Q.act, v, none) * (up * scale);
        }
        eight_store(static_cast<YT*>(Q.Y) + t * Q.ldy + rb * Q.R_u + i * EIGHT_ROWS + r, v);
    }
}

template <typename YT, int S, bool PAIR>
int launch_eight(const EightArgs& Q, hipStream_t st) {
    // Eight wavefronts where the row blocks are more than the CUs, so that they run at once: 344 of a pair, 16 tokens 14.6 us and 16.2 with sixteen.
    if (Q.T <= 32)
        return launch_pieces(Q.NB, 1024, [&](int64_t first, dim3 g) {
            if (Q.NB > 256) eight_kernel<YT, S, 1, 8, PAIR><<<g, dim3(512), 0, st>>>(Q, first);
            else eight_kernel<YT, S, 1, 16, PAIR><<<g, dim3(1024), 0, st>>>(Q, first);
        });
    constexpr int WR = 4;
    const int64_t row_tiles = tokens_in(Q.NB, PAIR ? WR : 2 * WR), tiles = row_tiles * tokens_in(Q.T, 64), few = Q.NB * tokens_in(Q.T, 64);
    if (!eight_few(few, tiles, PAIR) && fits_launch(tiles, WR * 64)) {
        eight_tiles_kernel<YT, S, WR, PAIR><<<dim3((uint32_t)tiles), dim3(WR * 64), 0, st>>>(Q, (uint32_t)row_tiles);
        return hipGetLastError() == hipSuccess ? WINDQ_OK : WINDQ_EHIP;
    }
    constexpr int WAVES = 8;
    return launch_pieces(few, WAVES * 64, [&](int64_t first, dim3 g) { eight_kernel<YT, S, 2, WAVES, PAIR><<<g, dim3(WAVES * 64), 0, st>>>(Q, first); });
}

template <typename YT, bool PAIR>
int launch_eight_steps(const EightArgs& Q, int S, hipStream_t st) {
    switch (S) {
        case 1: return launch_eight<YT, 1, PAIR>(Q, st);
        case 2: return launch_eight<YT, 2, PAIR>(Q, st);
        case 3: return launch_eight<YT, 3, PAIR>(Q, st);
        default: return launch_eight<YT, 4, PAIR>(Q, st);
    }
}

// ------------------------------------------------------------------------------------------------ checks
static bool chunk_ok(int64_t cols, int32_t chunk_w) { return cols > 0 && chunk_w >= 8 && chunk_w <= WINDQ_MAX_CHUNK && chunk_w % 8 == 0 && cols % chunk_w == 0 && cols <= MOST_SIDE; }

static int check_serving(const windq_serving* S, EightShape* E, EightPlan* P) {
    if (S == nullptr || S->image == nullptr || !aligned(S->image, 256)) return WINDQ_EINVAL;
    if (S->dtype != WINDQ_F32 && S->dtype != WINDQ_BF16) return WINDQ_EDTYPE;
    if (!chunk_ok(S->cols, S->chunk_w) || S->rows <= 0 || S->rows > MOST_SIDE || S->unit_rows < 0 || (S->unit_rows != 0 && S->rows % S->unit_rows != 0)) return WINDQ_ESHAPE;
    if (!sizes_fit(0, S->rows, S->cols, 0, 0)) return WINDQ_ESHAPE;
    *E = eight_shape(S->rows, S->cols, S->unit_rows == 0 ? S->rows : S->unit_rows, S->chunk_w);
    if (S->image_bytes > (size_t)EIGHT_MOST) return WINDQ_ESHAPE;
    if ((int64_t)S->image_bytes < E->header) return WINDQ_EINVAL;
    *P = {static_cast<const char*>(S->image), (int64_t)S->image_bytes, E->header};
    return WINDQ_OK;
}

static int product(const windq_serving* first, const windq_serving* second, const windq_tokens* X, int32_t act, void* Y, int32_t y_dtype, int64_t ld_y, void* stream) {
    EightArgs Q = {};
    EightShape E, other;
    int status = check_serving(first, &E, &Q.P[0]);
    if (status != WINDQ_OK) return status;
    if (second != nullptr) {
        status = check_serving(second, &other, &Q.P[1]);
        if (status != WINDQ_OK) return status;
        if (other.rows != E.rows || other.cols != E.cols || other.G != E.G || other.R_u != E.R_u) return WINDQ_ESHAPE;
        if (first->dtype != second->dtype) return WINDQ_EDTYPE;
    }
    if (X == nullptr) return WINDQ_EINVAL;
    if (y_dtype != WINDQ_F32 && y_dtype != WINDQ_BF16) return WINDQ_EDTYPE;
    if (X->cols != E.cols || X->chunk_w != E.G || X->tokens < 0) return WINDQ_ESHAPE;
    if (!sizes_fit(X->tokens, E.rows, E.cols, 0, 0) || !sizes_fit(X->tokens, E.rows, E.width, 0, 0)) return WINDQ_ESHAPE;
    if (ld_y < E.rows || ld_y > (int64_t)1 << 31) return WINDQ_ESHAPE;
    if (X->tokens == 0) return WINDQ_OK;
    if (X->codes == nullptr || X->scale == nullptr || X->sums == nullptr || Y == nullptr) return WINDQ_EINVAL;
    if (!aligned(X->codes, 16) || !aligned(X->scale, 4) || !aligned(X->sums, 16) || !aligned(Y, y_dtype == WINDQ_F32 ? 4 : 2)) return WINDQ_EINVAL;
    Q.codes = X->codes;
    Q.scale = X->scale;
    Q.sums = X->sums;
    Q.T = X->tokens;
    Q.Y = Y;
    Q.ldy = ld_y;
    Q.R_u = E.R_u;
    Q.RB = E.RB;
    Q.NB = E.NB;
    Q.width = E.width;
    Q.sums_ld = E.sums_ld;
    Q.affine = E.affine;
    Q.n_kb = E.n_kb;
    Q.act = act;
    Q.w_f32 = first->dtype == WINDQ_F32;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (second != nullptr) return y_dtype == WINDQ_F32 ? launch_eight_steps<float, true>(Q, E.S, st) : launch_eight_steps<uint16_t, true>(Q, E.S, st);
    return y_dtype == WINDQ_F32 ? launch_eight_steps<float, false>(Q, E.S, st) : launch_eight_steps<uint16_t, false>(Q, E.S, st);
}

}  // namespace windq

using namespace windq;

extern "C" int64_t windq_tokens8_width(int64_t cols, int32_t chunk_w) { return chunk_ok(cols, chunk_w) ? eight_shape(1, cols, 1, chunk_w).width : 0; }
extern "C" int64_t windq_tokens8_sums(int64_t cols, int32_t chunk_w) { return chunk_ok(cols, chunk_w) ? eight_shape(1, cols, 1, chunk_w).sums_ld : 0; }

extern "C" int windq_tokens8(const windq_mat* X, int32_t chunk_w, int8_t* codes, float* scale, int32_t* sums, void* stream) {
    if (X == nullptr) return WINDQ_EINVAL;
    const int status = check_tokens(X, X->cols, true);
    if (status != WINDQ_OK) return status;
    if (!chunk_ok(X->cols, chunk_w)) return WINDQ_ESHAPE;
    const EightShape E = eight_shape(1, X->cols, 1, chunk_w);
    if (!sizes_fit(X->rows, 1, E.width, 0, 0)) return WINDQ_ESHAPE;
    if (X->rows == 0) return WINDQ_OK;
    if (codes == nullptr || scale == nullptr || sums == nullptr) return WINDQ_EINVAL;
    if (!aligned(codes, 16) || !aligned(scale, 4) || !aligned(sums, 16)) return WINDQ_EINVAL;
    const TokensArgs Q = {X->data, X->ld, X->rows, codes, scale, sums, chunk_w, E.per_chunk * E.S * 4, E.S * 4, E.width / 8, E.sums_ld, E.n_kb};
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int launched = X->dtype == WINDQ_F32 ? launch_tokens8<float>(Q, st) : launch_tokens8<uint16_t>(Q, st);
    if (launched != WINDQ_OK || E.n_kb <= TOKENS_SUMS) return launched;
    return launch_pieces(tokens_in(X->rows * E.sums_ld, 256), 256, [&](int64_t first, dim3 g) { tokens8_sums_kernel<<<g, dim3(256), 0, st>>>(Q, first); });
}

extern "C" int windq_serving_layout(const uint8_t* action, int64_t rows, int64_t cols, int32_t chunk_w, int64_t unit_rows, int32_t dtype, int64_t* image_off) {
    if (action == nullptr || image_off == nullptr) return WINDQ_EINVAL;
    if (dtype != WINDQ_F32 && dtype != WINDQ_BF16) return WINDQ_EDTYPE;
    if (!chunk_ok(cols, chunk_w) || rows <= 0 || rows > MOST_SIDE || unit_rows < 0 || (unit_rows != 0 && rows % unit_rows != 0) || !sizes_fit(0, rows, cols, 0, 0)) return WINDQ_ESHAPE;
    const EightShape E = eight_shape(rows, cols, unit_rows == 0 ? rows : unit_rows, chunk_w);
    int64_t at = E.header;
    for (int64_t u = 0; u < E.U; ++u) {
        if (action[u] >= WINDQ_N_ACTIONS) return WINDQ_EINVAL;
        image_off[u] = at;
        at += eight_bytes(eight_kind(action[u]), E.S, dtype == WINDQ_F32) * E.RB * E.per_chunk;
    }
    image_off[E.U] = at + EIGHT_PAST;
    if (image_off[E.U] > EIGHT_MOST) return WINDQ_ESHAPE;
    return WINDQ_OK;
}

extern "C" int windq_serving_lay(const windq_packed* P, const int64_t* image_off, void* image, size_t image_bytes, void* stream) {
    PackArgs A = {};
    const int status = check_packed(P, &A);
    if (status != WINDQ_OK) return status;
    if (A.mask != nullptr || image_off == nullptr || image == nullptr || !aligned(image_off, 8) || !aligned(image, 256)) return WINDQ_EINVAL;
    if (!sizes_fit(0, A.rows, A.cols, 0, 0)) return WINDQ_ESHAPE;
    const EightShape E = eight_shape(A.rows, A.cols, A.R_u, A.G);
    if (image_bytes > (size_t)EIGHT_MOST) return WINDQ_ESHAPE;
    if ((int64_t)image_bytes < E.header) return WINDQ_EWORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return launch_pieces(tokens_in(E.U * E.RB * E.per_chunk, 4), 256,
                         [&](int64_t first, dim3 g) { serving_lay_kernel<<<g, dim3(256), 0, st>>>(A, E, image_off, static_cast<char*>(image), (int64_t)image_bytes, first); });
}

extern "C" int windq_project8(const windq_serving* P, const windq_tokens* X, void* Y, int32_t y_dtype, int64_t ld_y, void* stream) {
    return product(P, nullptr, X, WINDQ_SILU, Y, y_dtype, ld_y, stream);
}

extern "C" int windq_gated8(const windq_serving* gate, const windq_serving* up, const windq_tokens* X, int32_t act, void* H, int32_t h_dtype, int64_t ld_h, void* stream) {
    if (up == nullptr || act < WINDQ_SILU || act > WINDQ_GELU_TANH) return WINDQ_EINVAL;
    return product(gate, up, X, act, H, h_dtype, ld_h, stream);
}
