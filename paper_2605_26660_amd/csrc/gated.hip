// windq_gated: a batch of tokens through a pair of packed matrices, gate and up, of which act(gate) * up is kept; and its way back.
//   G[t] = w_gate x_t,   U[t] = w_up x_t,   H[t] = act(G[t]) * U[t]
//   dG = dH U act'(G),   dU = dH act(G),    dX[t] = w_gate^T dG[t] + w_up^T dU[t]
#include <math.h>

#include "windq_dx.hpp"
#include "windq_pair_few.hpp"
#include "windq_pair_gemm.hpp"
#include "windq_project_any.hpp"

namespace windq {

// Many bfloat16 tokens: the matrices are reconstructed in half precision, once a call, and multiplied by a plain product (windq_gemm.hpp).  Both factors have 11 bits of
// significand, and powers of two for a token and for a row that bring them below 2^15, so that what lies 2^28 below the largest of them still has all of its
// digits: the weights' rounding (tokens have none: bfloat16's eight bits fit) is eight times as fine as G's and U's own.
// From 65 tokens on, unless the kernel for few tokens has them all in one round of workgroups: 11008 x 4096, 128 tokens 84 us (by it some 130), 64 tokens 83 and 69 by it; 4096 x 4096, 128 tokens
// 57 and 38 by it (one round), 192 tokens 56 and 148; unpacking for every 128 tokens anew (as fp32 calls do) 118, 97 and 105.
constexpr int64_t GATED_MANY = PROJECT_FEW;
inline bool gated_few(const PackArgs& P, const PackArgs& up, int64_t T) {
    return (T <= PROJECT_FEW || tokens_in(P.rows, PF_ROWS) * tokens_in(T, 64) <= 256) && few_fits(P, T) && few_fits(up, T);
}

struct GatedWs {
    size_t planes, frag, few_xs, fields[2], unit[2], xs, beta[2], alpha[2], w, x, by_token, by_row, total;
};

// Rows of both matrices, 32 and 32 in turn, filled up to whole tiles.
inline int64_t gated_rows(int64_t rows) { return ((rows + 31) / 32 * 64 + GM_MOST - 1) / GM_MOST * GM_MOST; }

GatedWs gated_ws(int32_t dtype, int64_t T, int64_t rows, int64_t cols, int32_t G) {
    GatedWs w;
    size_t at = 0;
    auto take = [&at](size_t bytes) {
        const size_t here = at;
        at += round_up(bytes, 256);
        return here;
    };
    w.planes = take(dtype == WINDQ_F32 ? (size_t)(3 * T * cols) * 2 : 0);
    const bool few = dtype == WINDQ_BF16;                   // fewer tokens than asked for fit too
    const int64_t few_tokens = T < few_most(rows, cols, G) ? tokens_in(T, 64) * 64 : few_most(rows, cols, G);
    w.frag = take(few ? (size_t)cols * (size_t)few_tokens * 2 : 0);
    w.few_xs = take(few ? (size_t)(cols / 64 + 1) * (size_t)few_tokens * 4 : 0);
    const bool many = dtype == WINDQ_F32 && T > PROJECT_FEW;
    w.xs = take(many ? (size_t)(cols / 64) * (size_t)T * 16 : 0);
    for (int m = 0; m < 2; ++m) {
        w.fields[m] = take(many ? (size_t)(rows * cols) / (G == 128 || G == 96 || G == 64 ? 2 : 1) : 0);
        w.unit[m] = take(many ? (size_t)((rows + PT_STRIP - 1) / PT_STRIP) * (size_t)(cols / 64) * sizeof(KbWord) : 0);
        w.beta[m] = take(many ? (size_t)(cols / 64) * (size_t)rows * 16 : 0);
        w.alpha[m] = take(many ? (size_t)(cols / G) * (size_t)rows * 4 : 0);
    }
    const bool halves = few && T > GATED_MANY;
    w.w = take(halves ? (size_t)gated_rows(rows) * (size_t)gemm_k(cols) * 2 : 0);
    w.x = take(halves ? (size_t)T * (size_t)gemm_k(cols) * 2 : 0);
    w.by_token = take(halves ? (size_t)T * 4 : 0);
    w.by_row = take(halves ? (size_t)gated_rows(rows) * 4 : 0);
    w.total = at == 0 ? 256 : at;
    return w;
}

struct HalvesArgs {
    PackArgs P[2];
    const uint16_t* X;
    int64_t ldx, K;
    uint16_t* x;               // [T][K]
    float* by_token;           // powers, and losses in them (with_loss)
    uint16_t* w;               // [rows of both in turn, 32 and 32][K]
    float* by_row;
};

// Workgroups ahead: 16 rows of a matrix, the longer ones; the others: a token.  A wavefront has a k-block of them at a time, of one treatment, a lane a row and a quarter of its
// columns; where chunks are not whole k-blocks or a mask lies over them 128 columns, a lane an octet of two rows: lanes of different treatments would take
// turns, each waiting for its codes.  The units' treatments and places are looked up once.  Bound by the stores (180 MB for a pair of 11008 x 4096, 35 us at a copy's rate) and by chains
// of loads ahead of them: 66 us; a lane an octet 79, with skip rows looked through by one lane each 82 either way.
constexpr int HALVES_UNITS = 512, HALVES_ROWS = 16;

template <bool KNOWN, int O>                               // units of whole blocks of rows, and few enough of them in a row; O: chunks of one or more 32 O columns, no mask, or 0
__global__ __launch_bounds__(256) void gated_halves_kernel(const HalvesArgs Q, const int64_t first) {
    __shared__ float most[4][HALVES_ROWS], losses[4][HALVES_ROWS];
    __shared__ uint16_t trits_of[256];
    __shared__ uint64_t units[HALVES_UNITS];
    const int64_t blocks = (Q.P[0].rows + HALVES_ROWS - 1) / HALVES_ROWS, block = first + blockIdx.x, id = block - 2 * blocks;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (id >= 0) {
        const uint16_t* __restrict__ const x = Q.X + id * Q.ldx;
        float m = 0.0f, lost = 0.0f;
        for (int64_t c = threadIdx.x * 8; c < Q.P[0].cols; c += 2048) {
            float v[8];
            load8(x + c, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) m = finite_max(m, v[i]);
        }
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
        if (lane == 0) most[wave][0] = m;
        __syncthreads();
        m = fmaxf(fmaxf(most[0][0], most[1][0]), fmaxf(most[2][0], most[3][0]));
        const float by = power_below(m);
        const bool narrow = by >= 0x1p-16f;                 // no value becomes zero, and 8 bits are all there from 2^-14 on
        for (int64_t c = threadIdx.x * 8; c < Q.K; c += 2048) {
            float v[8] = {};
            if (c < Q.P[0].cols) load8(x + c, v);
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float y = v[i] * by;
                w[i] = half_bits<_Float16>(y);
                lost += narrow ? fabsf(y - (float)(_Float16)y) * 0x1p25f : half_lost(v[i], y);
            }
            *reinterpret_cast<uint4*>(Q.x + id * Q.K + c) = pack8(w);
        }
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) lost += __shfl_xor(lost, d, 64);
        if (lane == 0) losses[wave][0] = lost;
        __syncthreads();
        if (threadIdx.x == 0) Q.by_token[id] = m > 0.0f ? with_loss(1.0f / by, losses[0][0] + losses[1][0] + losses[2][0] + losses[3][0]) : power_of_nothing();
        return;
    }
    trits_of[threadIdx.x] = (uint16_t)trit_fields(threadIdx.x);
    const int mat = block >= blocks ? 1 : 0;
    const PackArgs& P = Q.P[mat];
    const int64_t r0 = (block - mat * blocks) * HALVES_ROWS, at = (r0 >> 5) * 64 + mat * 32 + (r0 & 31), rb = r0 / P.R_u;
    if constexpr (KNOWN)
        for (int32_t j = threadIdx.x; j < P.n_chunks; j += 256) {
            int64_t base;
            const int a = pk_action(P, rb * P.n_chunks + j, base);
            units[j] = (uint64_t)a << 56 | (uint64_t)(a == 0 ? 0 : base);
        }
    // A row's groups by sixteen threads: group(treatment, number) for those of codes, weight(value) for what stays as it is.
    const int64_t row = r0 + (threadIdx.x & 15);
    auto look = [&](auto group, auto weight) {
        auto weights = [&](int64_t j, int32_t first, int32_t step) {
#pragma unroll 2
            for (int32_t c = first; c < P.G; c += step) {
                float w[8];
                skip_row(P, row, j * P.G + c, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) weight(w[i]);
            }
        };
        if (row >= P.rows) return;
        if constexpr (KNOWN) {                              // rows of skip units by all threads: one that looks through 128 weights by itself takes as long as all the rest
            const int64_t g0 = rb * P.n_chunks * P.R_u + row - rb * P.R_u;
            for (int32_t j = threadIdx.x >> 4; j < P.n_chunks; j += 16)
                if (const int a = (int)(units[j] >> 56); a != 0) group(a, g0 + j * P.R_u);
            for (int32_t j = 0; j < P.n_chunks; ++j)
                if ((units[j] >> 56) == 0) weights(j, (int32_t)(threadIdx.x >> 4) * 8, 128);
        } else {
            const int64_t own = row / P.R_u;
            for (int64_t j = threadIdx.x >> 4; j < P.n_chunks; j += 16) {
                const int64_t u = own * P.n_chunks + j;
                int64_t base;
                const int a = pk_action(P, u, base);
                if (a != 0) group(a, u * P.R_u + row - own * P.R_u);
                else weights(j, 0, 8);
            }
        }
    };
    // the rows' largest magnitudes, and the smallest that half precision may take something from
    float m = 0.0f, least_group = 3.40282347e38f, least_weight = least_group;
    if constexpr (KNOWN) __syncthreads();
    look(
        [&](int a, int64_t g) {
            const float top = affine_top(P, a, g);
            m = fmaxf(m, top);
            least_group = top > 0.0f && top < least_group ? top : least_group;
        },
        [&](float w) {
            m = finite_max(m, w);
            least_weight = w != 0.0f && fabsf(w) < least_weight ? fabsf(w) : least_weight;
        });
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    if (lane < HALVES_ROWS) most[wave][lane] = m;
    __syncthreads();
    auto most_of = [&](int r) { return fmaxf(fmaxf(most[0][r], most[1][r]), fmaxf(most[2][r], most[3][r])); };
    auto power_of = [&](int r) { return power_below(most_of(r)); };
    {
        const float by = power_of(threadIdx.x & 15);
        float lost = 0.0f;
        if (__any(least_group * by < HALF_GROUP || least_weight * by < HALF_NORMAL)) {         // rare
            look([&](int a, int64_t g) { lost += P.G * group_lost(P, a, g, by); }, [&](float w) { lost += half_lost(w, w * by); });
            lost += __shfl_xor(lost, 32, 64);
            lost += __shfl_xor(lost, 16, 64);
        }
        if (lane < HALVES_ROWS) losses[wave][lane] = lost;
        __syncthreads();
        if (threadIdx.x < HALVES_ROWS && row < P.rows)
            Q.by_row[at + threadIdx.x] =
                most_of(threadIdx.x) > 0.0f ? with_loss(1.0f / by, losses[0][threadIdx.x] + losses[1][threadIdx.x] + losses[2][threadIdx.x] + losses[3][threadIdx.x]) : power_of_nothing();
    }
    if constexpr (O > 0) {
        // 16 rows by 32 O columns a wavefront at a time, a lane a row and O octets of it, whose codes are one load; they leave through LDS by whole lines
        constexpr int COLS = 32 * O, LD = 4 * O + 1;        // a row's sixteens of bytes in LDS
        __shared__ uint4 turned[4][16 * LD];
        const int sub = lane & 15, q = lane >> 4;
        const float by = power_of(sub);
        const int32_t there = P.rows - r0 < HALVES_ROWS ? (int32_t)(P.rows - r0) : HALVES_ROWS;
        const uint32_t lr = (uint32_t)(sub < there ? sub : there - 1);
        uint4* const mine = turned[wave];
        const int32_t per_chunk = P.G / COLS;
        const uint32_t lrow0 = (uint32_t)(r0 - rb * P.R_u);
        for (int32_t kb = wave; kb < (int32_t)(P.cols / COLS); kb += 4) {
            const int32_t j = kb / per_chunk, c = kb - j * per_chunk;
            const uint64_t unit = units[j];
            const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(unit >> 32)), lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)unit);
            const int kind = (int)(hi >> 24);
            const uint32_t bpg = (uint32_t)pk_bytes_per_group(kind, P.G);
            const uint8_t* const codes = P.codes + (((uint64_t)(hi & 0xffffffu) << 32 | lo) + (uint64_t)lrow0 * bpg);
            const int64_t g = (rb * P.n_chunks + j) * P.R_u + lrow0;
            const float scale = (P.scale + g)[lr] * by, offset = (P.offset + g)[lr] * by;
            const uint32_t first = (uint32_t)c * COLS + q * (8 * O), row_at = lr * bpg;
            uint4 w[O];
            switch (kind) {
                case 1: pair_fields<O, 8, true>(codes + (row_at + first), w); break;
                case 2: pair_fields<O, 4, true>(codes + (row_at + (first >> 1)), w); break;
                case 3: pair_fields<O, 3, true>(codes + (row_at + (first >> 3) * 3), w); break;
                case 4: pair_fields<O, 2, true>(codes + (row_at + (first >> 2)), w); break;
                case 5: {
                    const uint32_t k = first / 5u, from = k < bpg - 8u ? k : bpg - 8u;       // eight bytes within the row
                    pair_trits<O, true>(codes + (row_at + from), first - from * 5u, trits_of, w);
                    break;
                }
                case 6: pair_fields<O, 1, true>(codes + (row_at + (first >> 3)), w); break;
                default: {
#pragma unroll
                    for (int s = 0; s < O; ++s) {
                        float v[8];
                        skip_row(P, r0 + lr, (int64_t)kb * COLS + q * (8 * O) + s * 8, v);
                        w[s] = make_uint4(half_pair(v[0] * by, v[1] * by), half_pair(v[2] * by, v[3] * by), half_pair(v[4] * by, v[5] * by), half_pair(v[6] * by, v[7] * by));
                    }
                }
            }
            if (kind != 0) {
                const float b = fmaf(-pk_f0(kind), scale, kind >= 5 ? 0.0f : offset);
#pragma unroll
                for (int s = 0; s < O; ++s) w[s] = half_weights(w[s], scale, b);
            }
#pragma unroll
            for (int s = 0; s < O; ++s) mine[sub * LD + q * O + s] = w[s];
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (int i = 0; i < O; ++i) {
                const int n = (i * 64 + lane) / (4 * O), slot = i * 64 + lane - n * (4 * O);
                if (n < there) *reinterpret_cast<uint4*>(Q.w + (at + n) * Q.K + (int64_t)kb * COLS + slot * 8) = mine[n * LD + slot];
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
        for (int32_t c = (int32_t)P.cols + (int)(threadIdx.x >> 4) * 8; c < Q.K; c += 128)         // columns up to a whole step of the product
            if (sub < there) *reinterpret_cast<uint4*>(Q.w + (at + sub) * Q.K + c) = make_uint4(0u, 0u, 0u, 0u);
        return;
    }
    const int octet = wave & 1, part = octet * 4 + (lane >> 4);
    const float by[2] = {power_of(part * 2), power_of(part * 2 + 1)};
    const int64_t here = r0 + part * 2;
    if (here >= P.rows) return;                             // rows come in eights
    for (int64_t c = (wave >> 1) * 128 + (lane & 15) * 8; c < Q.K; c += 256) {
        uint32_t w[2][4] = {};
        auto put = [&](int i, int k, float v) {
            const uint32_t b = half_bits<_Float16>(v * by[i]);
            w[i][k >> 1] = (k & 1) != 0 ? w[i][k >> 1] | b << 16 : b;
        };
        if (c < P.cols) {
            const uint32_t j = (uint32_t)c / (uint32_t)P.G;
            if constexpr (KNOWN) {
                const uint64_t unit = units[j];
                rows_of<2>(P, here, c, rb * P.n_chunks + j, here - rb * P.R_u, ((int)c - (int)j * P.G) >> 3, (int)(unit >> 56), (int64_t)(unit & 0xffffffffffffffull), trits_of, put);
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float v[8];
                    weight_octet(P, here + i, c, trits_of, v);
#pragma unroll
                    for (int k = 0; k < 8; ++k) put(i, k, v[k]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) *reinterpret_cast<uint4*>(Q.w + (at + part * 2 + i) * Q.K + c) = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
    }
}

int launch_gated_halves(const ProjectArgs& Q, char* ws, const GatedWs& at, hipStream_t st) {
    const int64_t K = gemm_k(Q.P.cols), rows = gated_rows(Q.P.rows), tall = tokens_in(Q.T, GM_N);
    const HalvesArgs H = {{Q.P, Q.pair.up}, Q.X, Q.ldx, K, reinterpret_cast<uint16_t*>(ws + at.x), reinterpret_cast<float*>(ws + at.by_token),
                          reinterpret_cast<uint16_t*>(ws + at.w), reinterpret_cast<float*>(ws + at.by_row)};
    const bool mask = Q.P.mask != nullptr || Q.pair.up.mask != nullptr;
    const bool known = (Q.P.R_u == Q.P.rows || Q.P.R_u % HALVES_ROWS == 0) && Q.P.n_chunks <= HALVES_UNITS;
    const int status = launch_pieces(Q.T + 2 * tokens_in(Q.P.rows, HALVES_ROWS), 256, [&](int64_t first, dim3 g) {
        if (known && !mask && Q.P.G % 128 == 0) gated_halves_kernel<true, 4><<<g, dim3(256), 0, st>>>(H, first);
        else if (known && !mask && Q.P.G == 96) gated_halves_kernel<true, 3><<<g, dim3(256), 0, st>>>(H, first);
        else if (known && !mask && Q.P.G == 64) gated_halves_kernel<true, 2><<<g, dim3(256), 0, st>>>(H, first);
        else if (known) gated_halves_kernel<true, 0><<<g, dim3(256), 0, st>>>(H, first);
        else gated_halves_kernel<false, 0><<<g, dim3(256), 0, st>>>(H, first);
    });
    if (status != WINDQ_OK) return status;
    const int64_t by = rows / 256 * tall >= GM_TILES ? 256 : 128, large = rows / GM_MOST * tokens_in(Q.T, GW_N);
    const bool wide = gemm_wide(large, rows / by * tall, by);
    const int64_t tiles = wide ? large : rows / by * tall;
    GemmArgs M = {};
    M.wt = H.w;
    M.dY = H.x;
    M.ldy = K;
    M.K = (int32_t)K;
    M.T = Q.T;
    M.cols = rows;
    M.dX = static_cast<uint16_t*>(Q.Y);
    M.ldx = Q.ldy;
    M.col_blocks = (uint32_t)(rows / (wide ? GM_MOST : by));
    M.tiles = (int32_t)tiles;
    M.each = (int32_t)(K / GM_K);
    M.by_token = H.by_token;
    M.by_row = H.by_row;
    M.gate = Q.P;
    M.pair = Q.pair;
    M.raw = Q.X;
    M.ld_raw = Q.ldx;
    // tiles are no more than 2^31 / (64 x 128) and two sides' edges: one launch holds them
    if (wide) pair_gemm_kernel<<<dim3((uint32_t)tiles), dim3(GW_THREADS), 0, st>>>(M);
    else if (by == 256) dx_gemm_kernel<4, true, true><<<dim3((uint32_t)tiles), dim3(GM_THREADS), 0, st>>>(M);
    else dx_gemm_kernel<2, true, true><<<dim3((uint32_t)tiles), dim3(GM_THREADS), 0, st>>>(M);
    return hipGetLastError() == hipSuccess ? WINDQ_OK : WINDQ_EHIP;
}

template <int S>
int launch_gated_tiles(const ProjectArgs& Q, char* ws, const GatedWs& at, hipStream_t st) {
    TileArgs A = {};
    A.P = Q.P;
    A.X = Q.X;
    A.ldx = Q.ldx;
    A.plane = Q.plane;
    A.raw = Q.raw;
    A.ld_raw = Q.ld_raw;
    A.T = Q.T;
    A.Y = Q.Y;
    A.ldy = Q.ldy;
    A.xs = reinterpret_cast<uint4*>(ws + at.xs);
    A.unit_fields = Q.P.R_u * Q.P.G / (tile_natural(Q.P.G, S) ? 2 : 1);
    A.n_kb = (int32_t)(Q.P.cols / (16 * S));
    A.row_blocks = (uint32_t)((Q.P.rows + PT_ROWS / 2 - 1) / (PT_ROWS / 2));
    A.pair = Q.pair;
    auto matrix = [&](int m) {
        A.fields = reinterpret_cast<uint8_t*>(ws + at.fields[m]);
        A.unit = reinterpret_cast<KbWord*>(ws + at.unit[m]);
        A.beta = reinterpret_cast<uint4*>(ws + at.beta[m]);
        A.alpha = reinterpret_cast<float*>(ws + at.alpha[m]);
    };
    const int64_t strips = (Q.P.rows / Q.P.R_u) * Q.P.n_chunks * ((Q.P.R_u + PT_STRIP - 1) / PT_STRIP);
    for (int m = 1; m >= 0; --m) {                          // the sums of X with the gate's
        matrix(m);
        A.P = m == 1 ? Q.pair.up : Q.P;
        const int64_t wgs = strips + (m == 0 ? tokens_in(A.n_kb * Q.T, PT_SUMS) : 0);
        const int status = launch_pieces(wgs, 256, [&](int64_t first, dim3 g) { tiles_prepare_kernel<float, S><<<g, dim3(256), 0, st>>>(A, strips, first); });
        if (status != WINDQ_OK) return status;
    }
    A.unit_up = reinterpret_cast<KbWord*>(ws + at.unit[1]);
    A.beta_up = reinterpret_cast<uint4*>(ws + at.beta[1]);
    // tiles are no more than 2^31 / (64 x 128) and two sides' edges: one launch holds them
    const int64_t tiles = (int64_t)A.row_blocks * ((Q.T + PT_TOKENS - 1) / PT_TOKENS);
    project_tiles_kernel<float, S, true><<<dim3((uint32_t)tiles), dim3(PT_THREADS), 0, st>>>(A);
    return hipGetLastError() == hipSuccess ? WINDQ_OK : WINDQ_EHIP;
}

// fp32: 16 rows by 16 tokens a workgroup up to so many tiles of 128 rows of both by 128 tokens, whose time is a round's until the CUs are full.  1024 x 4096, 300 tokens (24
// tiles) 182 us (plans of all treatments alike), tiles some 490; 2048 x 2048, 300 tokens (48) 158 and 300, 1000 tokens (128) 472 and 300; 1024 x 4096, 1000 tokens (64) 520 and 493; 1000 x 1056, 1000 tokens (64)
// 126 and 154; 4096 x 1024, 300 tokens (96) 211 and 164.
constexpr int64_t PAIR_TILES = 64;

template <typename XT>
int gated_all(ProjectArgs& Q, const windq_mat* X, char* ws, const GatedWs& at, hipStream_t st) {
    const int64_t T = Q.T;
    if constexpr (sizeof(XT) == 4) {
        uint16_t* planes = reinterpret_cast<uint16_t*>(ws + at.planes);
        const int status = launch_planes(static_cast<const float*>(X->data), X->ld, T, (int32_t)Q.P.cols, planes, st);
        if (status != WINDQ_OK) return status;
        Q.X = planes;
        Q.ldx = Q.P.cols;
        Q.plane = T * Q.P.cols;
    } else {
        if (gated_few(Q.P, Q.pair.up, T)) {
            FewArgs F = {Q.P, Q.X, Q.ldx, T, static_cast<uint16_t*>(Q.Y), Q.ldy, nullptr, Q.A, 0, reinterpret_cast<uint4*>(ws + at.frag), reinterpret_cast<float*>(ws + at.few_xs), 0, 0, 0, 0, Q.pair};
            const int steps = Q.P.G % 128 == 0 ? 8 : Q.P.G / 16;
            F.n_kb = (int32_t)(Q.P.cols / (16 * steps));
            if (T <= PAIR_FEW) {
                F.raw = Q.raw;
                F.ld_raw = Q.ld_raw;
                return launch_pair_few<uint16_t>(F, st);
            }
            return steps == 8 ? launch_few<8, true>(F, nullptr, st) : (steps == 6 ? launch_few<6, true>(F, nullptr, st) : launch_few<4, true>(F, nullptr, st));
        }
    }
    const bool mask = Q.P.mask != nullptr || Q.pair.up.mask != nullptr;
    if constexpr (sizeof(XT) == 2) {
        if (T > GATED_MANY && Q.P.rows % 8 == 0) return launch_gated_halves(Q, ws, at, st);
    } else {
        const int S = !mask && T > PROJECT_FEW && (Q.P.rows + 15) / 16 * tokens_in(T, 64) > 512 ? tile_steps(Q.P) : 0;
        if (pair_fits(Q.P) && pair_fits(Q.pair.up) && fits_launch(tokens_in(Q.P.rows, PR_ROWS) * tokens_in(T, 16), 512) && (S == 0 || tokens_in(Q.P.rows, PT_ROWS / 2) * tokens_in(T, PT_TOKENS) <= PAIR_TILES)) {
            FewArgs F = {};
            F.P = Q.P;
            F.X = Q.X;
            F.ldx = Q.ldx;
            F.T = T;
            F.Y = static_cast<uint16_t*>(Q.Y);
            F.ldy = Q.ldy;
            F.pair = Q.pair;
            F.plane = Q.plane;
            F.raw = Q.raw;
            F.ld_raw = Q.ld_raw;
            return launch_pair_few<float>(F, st);
        }
        if (S == 8) return launch_gated_tiles<8>(Q, ws, at, st);
        if (S == 6) return launch_gated_tiles<6>(Q, ws, at, st);
        if (S == 4) return launch_gated_tiles<4>(Q, ws, at, st);
    }
    return mask ? launch_project_any<XT, true, true>(Q, st) : launch_project_any<XT, false, true>(Q, st);
}

// Two packed matrices of one shape, chunk width, units and weight type.
int check_pair(const windq_packed* gate, const windq_packed* up, PackArgs* A, PackArgs* B) {
    int status = check_packed(gate, A);
    if (status == WINDQ_OK) status = check_packed(up, B);
    if (status != WINDQ_OK) return status;
    if (A->rows != B->rows || A->cols != B->cols || A->G != B->G || A->R_u != B->R_u) return WINDQ_ESHAPE;
    return A->w_f32 != B->w_f32 ? WINDQ_EDTYPE : WINDQ_OK;
}

// ------------------------------------------------------------------------------------------------ the way back
// dX is one product whose sum runs along the gate's rows and then the up's.  In bfloat16 calls both factors are half precision numbers: 11 bits of
// significand, where bfloat16's 8 would be as coarse as dX's own rounding three times over (dX 1.7 times as far off as its rounding alone).  Their
// range is what powers of two make of it: a token's dG and dU, and a chunk's weights in both matrices, are brought below 2^15, and what lies 2^28 below the
// largest of them still has all of its digits.  The powers come off dX in fp32.  What lies lower is counted as lost, token by token and octet of columns by octet, and a value of dX
// that it could change by 2^-10 is formed again from dH, G, U and the weights in fp64 (dx_again), by the product or by the join of its parts.
//   The launch ahead: a workgroup a token (dG, dU and, from them, the token's power: what an activation shuts out has no part in it), and
// workgroups of 512 rows by one chunk (the largest magnitude their groups can take).  Then the reconstruction, turned, then the product.
constexpr int RANGE_ROWS = 512;

struct SlopeArgs {
    const void* dH;
    const void* G;
    const void* U;
    int64_t ld_dh, ld_save, T, rows;
    int32_t act;
    void* dG;                  // the caller's, or null
    void* dU;
    int64_t ld_d;
    void* to;                  // bfloat16 calls: [T][2 K] in half precision; fp32: [2][T][K]; or null: dX is not wanted
    int64_t K;
    float* by_token;           // powers, and losses in them (with_loss)
    bool wide;                 // all rows of all tensors on 16 bytes
    PackArgs P[2];
    float2* range;             // [chunks][2][strips]
    int32_t strips;
    int64_t ranges;            // workgroups for them
    int32_t* lost_octet;       // counted by the next launch, zeros so far
    uint32_t* there_octet;     // as well
    int64_t octets;
};

template <typename XT>
__device__ __forceinline__ void load_octet(const XT* __restrict__ p, int64_t left, bool wide, float (&v)[8]) {
    if (wide && left >= 8) return load8(p, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = 0.0f;
        if (i < left) {
            if constexpr (sizeof(XT) == 4) v[i] = p[i];
            else v[i] = bf16_bits_to_f32(p[i]);
        }
    }
}

template <typename XT>
__device__ __forceinline__ void store_octet(XT* __restrict__ p, int64_t left, bool wide, const float (&v)[8]) {
    if (wide && left >= 8) {
        if constexpr (sizeof(XT) == 4) {
            reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = f32_to_bf16_bits(v[i]);
            *reinterpret_cast<uint4*>(p) = pack8(w);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) store_y(p + i, v[i]);
}

// PER octets of dG and of dU a thread, kept in registers from where they are formed, and stored for the caller, to where the token's power is put on (bfloat16 calls with whole
// octets in every row); 0: any number, formed twice.
template <typename XT, int PER, int THREADS>
__device__ __forceinline__ void slopes(const SlopeArgs& Q, int64_t t) {
    constexpr int STEP = THREADS * 8, WAVES = THREADS / 64;
    __shared__ float most[WAVES], losses[WAVES];
    const XT* __restrict__ const dh = static_cast<const XT*>(Q.dH) + t * Q.ld_dh;
    const XT* __restrict__ const g = static_cast<const XT*>(Q.G) + t * Q.ld_save;
    const XT* __restrict__ const u = static_cast<const XT*>(Q.U) + t * Q.ld_save;
    float by = 1.0f, m = 0.0f, lost = 0.0f;
    auto form = [&](const float (&a)[8], const float (&b)[8], const float (&c)[8], float (&dg)[8], float (&du)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float slope;
            const float y = activation<true>(Q.act, b[i], slope);
            dg[i] = a[i] * c[i] * slope;
            du[i] = a[i] * y;
        }
    };
    auto formed = [&](int64_t r, float (&dg)[8], float (&du)[8]) {
        float a[8] = {}, b[8] = {}, c[8] = {};
        const int64_t left = Q.rows - r;
        if (left > 0) {
            load_octet(dh + r, left, Q.wide, a);
            load_octet(g + r, left, Q.wide, b);
            load_octet(u + r, left, Q.wide, c);
        }
        form(a, b, c, dg, du);
    };
    auto larger = [&](const float (&dg)[8], const float (&du)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) m = finite_max(finite_max(m, dg[i]), du[i]);
    };
    auto power = [&] {
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
        if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < WAVES; ++k) m = fmaxf(m, most[k]);
        by = power_below(m);
    };
    auto power_with_loss = [&] {
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) lost += __shfl_xor(lost, d, 64);
        if ((threadIdx.x & 63) == 0) losses[threadIdx.x >> 6] = lost;
        __syncthreads();
        float all = 0.0f;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) all += losses[k];
        if (threadIdx.x == 0) Q.by_token[t] = m > 0.0f ? with_loss(1.0f / by, all) : power_of_nothing();
    };
    auto keep = [&](int64_t r, const float (&dg)[8], const float (&du)[8]) {
        const int64_t left = Q.rows - r;
        if (Q.dG == nullptr || left <= 0) return;
        store_octet(static_cast<XT*>(Q.dG) + t * Q.ld_d + r, left, Q.wide, dg);
        store_octet(static_cast<XT*>(Q.dU) + t * Q.ld_d + r, left, Q.wide, du);
    };
    auto hand_on = [&](int64_t r, const float (&dg)[8], const float (&du)[8]) {
        if constexpr (sizeof(XT) == 2) {
            uint16_t* const to = static_cast<uint16_t*>(Q.to) + t * 2 * Q.K + r;
            uint32_t w[2][8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[0][i] = half_bits<_Float16>(dg[i] * by);
                w[1][i] = half_bits<_Float16>(du[i] * by);
            }
            const uint4 a = pack8(w[0]), b = pack8(w[1]);
            *reinterpret_cast<uint4*>(to) = a;
            *reinterpret_cast<uint4*>(to + Q.K) = b;
            // seldom: a half below the normal numbers
            typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
            u16x2 least = {0x7fff, 0x7fff};
            for (uint32_t x : {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}) least = __builtin_elementwise_min(least, __builtin_bit_cast(u16x2, x & 0x7fff7fffu));
            if (r < Q.rows && (least[0] < 0x400 || least[1] < 0x400)) {
#pragma unroll
                for (int i = 0; i < 8; ++i) lost += half_lost(dg[i], dg[i] * by) + half_lost(du[i], du[i] * by);
            }
        } else {
            store_octet(static_cast<float*>(Q.to) + t * Q.K + r, 8, true, dg);
            store_octet(static_cast<float*>(Q.to) + (Q.T + t) * Q.K + r, 8, true, du);
        }
    };
    if constexpr (PER > 0) {
        uint4 held[PER][3];
        float dg[PER][8], du[PER][8];
        auto values = [](uint4 v, float (&x)[8]) {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (i & 1) != 0 ? __uint_as_float(w[i >> 1] & 0xffff0000u) : __uint_as_float(w[i >> 1] << 16);
        };
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int64_t r = threadIdx.x * 8 + k * STEP;
            const bool in = r < Q.rows;
            held[k][0] = in ? *reinterpret_cast<const uint4*>(dh + r) : make_uint4(0u, 0u, 0u, 0u);
            held[k][1] = in ? *reinterpret_cast<const uint4*>(g + r) : make_uint4(0u, 0u, 0u, 0u);
            held[k][2] = in ? *reinterpret_cast<const uint4*>(u + r) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            float a[8], b[8], c[8];
            values(held[k][0], a);
            values(held[k][1], b);
            values(held[k][2], c);
            form(a, b, c, dg[k], du[k]);
            larger(dg[k], du[k]);
            keep(threadIdx.x * 8 + k * STEP, dg[k], du[k]);
        }
        power();
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int64_t r = threadIdx.x * 8 + k * STEP;
            if (r < Q.K) hand_on(r, dg[k], du[k]);
        }
        power_with_loss();
    } else {
        if (sizeof(XT) == 2 && Q.to != nullptr) {
            for (int64_t r = threadIdx.x * 8; r < Q.rows; r += STEP) {
                float dg[8], du[8];
                formed(r, dg, du);
                larger(dg, du);
            }
            power();
        }
        for (int64_t r = threadIdx.x * 8; r < (Q.to != nullptr ? Q.K : Q.rows); r += STEP) {
            float dg[8], du[8];
            formed(r, dg, du);
            keep(r, dg, du);
            if (Q.to != nullptr) hand_on(r, dg, du);
        }
        if (sizeof(XT) == 2 && Q.to != nullptr) power_with_loss();
    }
}

// The largest finite magnitude that a weight of RANGE_ROWS rows of a chunk can have, and the smallest that half precision may take
// something from (group_range); the largest less than 0: there are codes.
template <int THREADS>
__device__ __forceinline__ void range_of(const SlopeArgs& Q, int64_t block) {
    constexpr int WAVES = THREADS / 64;
    __shared__ float most[WAVES], least[WAVES];
    const int m = (int)(block / ((int64_t)Q.strips * Q.P[0].n_chunks));
    const PackArgs& P = Q.P[m];
    const int64_t rest = block - (int64_t)m * Q.strips * P.n_chunks, j = rest / Q.strips, strip = rest - j * Q.strips;
    float most_here = 0.0f, least_here = 3.40282347e38f;
    bool coded = false;
    for (int k = threadIdx.x; k < RANGE_ROWS; k += THREADS) {
        const int64_t row = strip * RANGE_ROWS + k;
        if (row >= P.rows) break;
        group_range(P, row, j, most_here, least_here, coded);
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        most_here = fmaxf(most_here, __shfl_xor(most_here, d, 64));
        least_here = fminf(least_here, __shfl_xor(least_here, d, 64));
    }
    coded = __any(coded);
    if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = coded ? -most_here : most_here, least[threadIdx.x >> 6] = least_here;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < WAVES; ++k) most_here = fmaxf(most_here, fabsf(most[k])), least_here = fminf(least_here, least[k]), coded |= most[k] < 0.0f;
    if (threadIdx.x == 0) Q.range[(j * 2 + m) * Q.strips + strip] = make_float2(coded ? -most_here : most_here, least_here);
    if (block == 0)
        for (int64_t k = threadIdx.x; k < Q.octets; k += THREADS) Q.lost_octet[k] = 0, Q.there_octet[k] = 0;
}

template <typename XT, int PER = 0, int THREADS = 256>
__global__ __launch_bounds__(THREADS) void gated_slopes_kernel(const SlopeArgs Q, const int64_t first) {
    const int64_t block = first + blockIdx.x;               // the weights' ahead: those of skip units take long
    if (block < Q.ranges) range_of<THREADS>(Q, block);
    else slopes<XT, PER, THREADS>(Q, block - Q.ranges);
}

struct GatedTurnArgs {
    PackArgs P[2];
    int32_t K;
    uint16_t* wt;              // [cols][2 K]
    int64_t turns;             // workgroups of a matrix
    const float2* range;
    int32_t strips;
    float* by_octet;
    int32_t* lost_octet;
    uint32_t* there_octet;
};

template <bool PLAIN>
__global__ __launch_bounds__(256) void gated_turn_kernel(const GatedTurnArgs Q, const int64_t first) {
    const int64_t id = first + blockIdx.x;
    const int m = id >= Q.turns ? 1 : 0;
    const int64_t block = id - m * Q.turns;
    const int32_t row_blocks = (Q.K + 255) / 256;
    const int64_t cb = block / row_blocks, col = cb * 64 + (threadIdx.x >> 5) * 8;
    const PackArgs& P = Q.P[m];
    float most = 0.0f, least = 3.40282347e38f;
    bool coded = false;
    if (col < P.cols) {
        const float2* const range = Q.range + col / P.G * 2 * Q.strips;
        for (int32_t k = threadIdx.x & 31; k < 2 * Q.strips; k += 32) {
            const float2 r = range[k];
            most = fmaxf(most, fabsf(r.x)), least = fminf(least, r.y), coded |= r.x < 0.0f;
        }
    }
    coded = PLAIN && (uint32_t)(__ballot(coded) >> (threadIdx.x & 32)) != 0;
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) {
        most = fmaxf(most, __shfl_xor(most, d, 32));
        least = fminf(least, __shfl_xor(least, d, 32));
    }
    const float by = power_below(most);
    if (id - cb * row_blocks == 0 && (threadIdx.x & 31) == 0 && col < P.cols) Q.by_octet[col >> 3] = most > 0.0f ? with_codes(1.0f / by, coded) : power_of_nothing();
    if (least * by < HALF_GROUP && col < P.cols) {          // rare
        const int32_t lost = rows_lost(P, (block - cb * row_blocks) * 256 + (threadIdx.x & 31) * 8, col, by);
        if (lost != 0) atomicAdd(Q.lost_octet + (col >> 3), lost);
    }
    uint32_t there = turn<_Float16, PLAIN>(P, Q.K, 2 * (int64_t)Q.K, by, Q.wt + (int64_t)m * Q.K, block);
    if (PLAIN && !__any(there != 0)) return;                // columns of a chunk with codes are all there
#pragma unroll 1
    for (int d = 16; d >= 1; d >>= 1) there |= (uint32_t)__shfl_xor((int)there, d, 32);
    if ((threadIdx.x & 31) == 0 && there != 0) atomicOr(Q.there_octet + (col >> 3), there);
}

// The parts of dX added up, a thread per token and octet of columns; columns that lie too low are formed again.
struct GatedJoinArgs {
    GemmArgs M;
    int32_t splits;
};

__global__ __launch_bounds__(256) void gated_join_kernel(const GatedJoinArgs J, const int64_t first) {
    const GemmArgs& Q = J.M;
    const int lane = threadIdx.x & 63;
    const int64_t i = (first + blockIdx.x) * 256 + threadIdx.x, octets = Q.cols >> 3;
    const bool in = i < Q.T * octets;
    const int64_t t = in ? i / octets : Q.T - 1, o = in ? i - t * octets : 0, c = o * 8;
    const float by_token = Q.by_token[t], by_octet = Q.by_octet[o];
    const int32_t lost = Q.lost_octet[o];
    float v[8] = {};
#pragma unroll 4
    for (int32_t s = 0; s < J.splits; ++s) {
        float p[8];
        load8(Q.part + (s * Q.T + t) * Q.cols + c, p);
#pragma unroll
        for (int m = 0; m < 8; ++m) v[m] += p[m];
    }
    const float low = ldexpf(lost_below(by_token, by_octet, lost), exponent_of(by_token) + exponent_of(by_octet));
    const uint32_t there = has_codes(by_octet) || lost != 0 ? 0xffu : Q.there_octet[o];
    bool bad = false;
#pragma unroll
    for (int m = 0; m < 8; ++m) bad |= fabsf(v[m]) < low && (there >> m & 1u) != 0u;
#pragma unroll 1
    for (uint64_t left = __ballot(bad && in); left != 0; left &= left - 1) {
        const int which = __builtin_ctzll(left);
        const int64_t id = i - lane + which, token = id / octets;
        double sum[8];
        dx_again(Q.gate, Q.pair.up, Q.pair.act, Q.again, token, (id - token * octets) * 8, lane, sum);
#pragma unroll
        for (int m = 0; m < 8; ++m)
            if (lane == which && fabsf(v[m]) < low && (there >> m & 1u) != 0u) v[m] = (float)sum[m];
    }
    if (!in) return;
    uint16_t* __restrict__ const out = Q.dX + t * Q.ldx + c;
    uint32_t w[8];
#pragma unroll
    for (int m = 0; m < 8; ++m) w[m] = f32_to_bf16_bits(v[m]);
    if ((Q.ldx & 7) == 0 && (reinterpret_cast<uintptr_t>(Q.dX) & 15) == 0) {
        *reinterpret_cast<uint4*>(out) = pack8(w);
    } else {
#pragma unroll
        for (int m = 0; m < 8; ++m) out[m] = (uint16_t)w[m];
    }
}

struct GatedGradWs {
    size_t to, wt, gm, by_token, by_octet, lost_octet, there_octet, range, dxf, total;
    int64_t K;
};

GatedGradWs gated_grad_ws(int32_t dtype, int64_t T, int64_t rows, int64_t cols, int32_t G) {
    GatedGradWs w;
    const bool bf = dtype == WINDQ_BF16;
    w.K = bf ? gemm_k(rows) : in_eights(rows);
    size_t at = 0;
    auto take = [&at](size_t bytes) {
        const size_t here = at;
        at += round_up(bytes, 256);
        return here;
    };
    w.to = take((size_t)(2 * T * w.K) * (bf ? 2 : 4));
    w.wt = take(bf && T > 0 ? (size_t)gemm_cols(cols) * (size_t)(2 * w.K) * 2 : 0);
    w.gm = take(bf ? (size_t)gemm_parts(T, 2 * w.K, cols) * 4 : 0);
    w.by_token = take(bf ? (size_t)T * 4 : 0);
    w.by_octet = take(bf ? (size_t)(cols / 8 + 1) * 4 : 0);
    w.lost_octet = take(bf ? (size_t)(cols / 8 + 1) * 4 : 0);
    w.there_octet = take(bf ? (size_t)(cols / 8 + 1) * 4 : 0);
    w.range = take(bf ? (size_t)(cols / G + 1) * 2 * (size_t)tokens_in(rows, RANGE_ROWS) * 8 : 0);
    w.dxf = take(bf ? 0 : DXF_BYTES);
    w.total = at == 0 ? 256 : at;
    return w;
}

size_t gated_grad_ws_bytes(int32_t dtype, int64_t T, int64_t rows, int64_t cols, int32_t G) { return gated_grad_ws(dtype, T, rows, cols, G).total; }

template <typename XT>
int gated_grad_all(SlopeArgs& S, void* dX, int64_t ld_dx, char* ws, const GatedGradWs& at, hipStream_t st) {
    constexpr bool bf = sizeof(XT) == 2;
    const PackArgs& P = S.P[0];
    const int64_t T = S.T, cols = P.cols;
    int64_t ahead = T;
    if (dX != nullptr) {
        S.to = ws + at.to;
        S.K = at.K;
        if (bf) {
            S.by_token = reinterpret_cast<float*>(ws + at.by_token);
            S.range = reinterpret_cast<float2*>(ws + at.range);
            S.lost_octet = reinterpret_cast<int32_t*>(ws + at.lost_octet);
            S.there_octet = reinterpret_cast<uint32_t*>(ws + at.there_octet);
            S.octets = cols / 8;
            S.strips = (int32_t)tokens_in(P.rows, RANGE_ROWS);
            S.ranges = 2 * (int64_t)S.strips * P.n_chunks;
            ahead += S.ranges;
        }
    }
    const int64_t each = bf && dX != nullptr && S.wide && P.rows % 8 == 0 ? tokens_in(S.K, 2048) : 0;
    // An octet that is formed is 16 registers: as few of them a thread as leave no thread without.  11008 rows, 2048 tokens: three by 512 threads 74 us, six by 256 92; 4104 rows, 500
    // tokens: three by 256 12.5, two by 512 14.0; 13824 rows, 512 tokens: four by 512 34, formed twice (0) 41.
    int status = launch_pieces(ahead, 512, [&](int64_t first, dim3 g) {
        if constexpr (bf) {
            if (each == 1) return gated_slopes_kernel<XT, 1><<<g, dim3(256), 0, st>>>(S, first);
            if (each == 2) return gated_slopes_kernel<XT, 1, 512><<<g, dim3(512), 0, st>>>(S, first);
            if (each == 3) return gated_slopes_kernel<XT, 3><<<g, dim3(256), 0, st>>>(S, first);
            if (each == 4) return gated_slopes_kernel<XT, 2, 512><<<g, dim3(512), 0, st>>>(S, first);
            if (each == 5 || each == 6) return gated_slopes_kernel<XT, 3, 512><<<g, dim3(512), 0, st>>>(S, first);
            if (each == 7 || each == 8) return gated_slopes_kernel<XT, 4, 512><<<g, dim3(512), 0, st>>>(S, first);
        }
        gated_slopes_kernel<XT><<<g, dim3(256), 0, st>>>(S, first);
    });
    if (status != WINDQ_OK || dX == nullptr) return status;
    if constexpr (bf) {
        const int32_t K2 = (int32_t)(2 * at.K);
        const GatedTurnArgs R = {{S.P[0], S.P[1]}, (int32_t)at.K, reinterpret_cast<uint16_t*>(ws + at.wt), ((cols + 63) / 64) * ((at.K + 255) / 256), S.range, S.strips,
                                 reinterpret_cast<float*>(ws + at.by_octet), S.lost_octet, S.there_octet};
        const bool plain = P.mask == nullptr && S.P[1].mask == nullptr && P.rows % 8 == 0 && (P.R_u == P.rows || P.R_u % 8 == 0);
        status = launch_pieces(2 * R.turns, 256, [&](int64_t first, dim3 g) {
            if (plain) gated_turn_kernel<true><<<g, dim3(256), 0, st>>>(R, first);
            else gated_turn_kernel<false><<<g, dim3(256), 0, st>>>(R, first);
        });
        if (status != WINDQ_OK) return status;
        // tiles are no more than 2^31 / 128^2 and two sides' edges: one launch holds them
        const int64_t tall = tokens_in(T, GM_N), by = tokens_in(cols, 256) * tall >= GM_TILES ? 256 : 128, tiles = tokens_in(cols, by) * tall;
        GemmArgs M = {R.wt, static_cast<const uint16_t*>(S.to), K2, K2, T, cols, static_cast<uint16_t*>(dX), ld_dx, nullptr, nullptr, {}, (uint32_t)tokens_in(cols, by), nullptr,
                      (int32_t)tiles, K2 / GM_K, S.by_token, R.by_octet, S.P[0]};
        M.pair.up = S.P[1];
        M.pair.act = S.act;
        M.lost_octet = S.lost_octet;
        M.there_octet = S.there_octet;
        M.again = {static_cast<const uint16_t*>(S.dH), static_cast<const uint16_t*>(S.G), static_cast<const uint16_t*>(S.U), S.ld_dh, S.ld_save};
        if (by == 256) {
            dx_gemm_kernel<4, true><<<dim3((uint32_t)tiles), dim3(GM_THREADS), 0, st>>>(M);
            return hipGetLastError() == hipSuccess ? WINDQ_OK : WINDQ_EHIP;
        }
        const int32_t each = gemm_each(K2, tiles), splits = (int32_t)tokens_in(K2 / GM_K, each);
        if (splits > 1) {
            M.each = each;
            M.part = reinterpret_cast<float*>(ws + at.gm);
        }
        dx_gemm_kernel<2, true><<<dim3((uint32_t)(tiles * splits)), dim3(GM_THREADS), 0, st>>>(M);
        if (hipGetLastError() != hipSuccess) return WINDQ_EHIP;
        if (splits == 1) return WINDQ_OK;
        const GatedJoinArgs J = {M, splits};
        return launch_pieces(tokens_in(T * (cols / 8), 256), 256, [&](int64_t first, dim3 g) { gated_join_kernel<<<g, dim3(256), 0, st>>>(J, first); });
    } else {
        DxArgs Q = {};
        Q.P = P;
        Q.packed = true;
        Q.T = T;
        Q.dX = dX;
        Q.ldx = ld_dx;
        Q.dY = S.to;
        Q.ldy = at.K;
        Q.up = S.P[1];
        Q.dY_up = static_cast<float*>(S.to) + T * at.K;
        Q.part = reinterpret_cast<float*>(ws + at.dxf);
        return launch_dx_f32(Q, st);
    }
}

}  // namespace windq

using namespace windq;

extern "C" size_t windq_gated_workspace_bytes(int32_t grad, int32_t dtype, int64_t tokens, int64_t rows, int64_t cols, int32_t chunk_w) {
    if ((dtype != WINDQ_F32 && dtype != WINDQ_BF16) || tokens < 0 || rows <= 0 || cols <= 0 || chunk_w <= 0) return 0;
    if (!sizes_fit(tokens, rows, cols, 0, 0) || (grad != 0 && !grad_sizes_fit(tokens, rows, cols))) return 0;
    return grad != 0 ? gated_grad_ws_bytes(dtype, tokens, rows, cols, chunk_w) : gated_ws(dtype, tokens, rows, cols, chunk_w).total;
}

extern "C" int windq_gated(const windq_packed* gate, const windq_packed* up, const windq_mat* X, int32_t act, void* H, int64_t ld_h, void* G, void* U,
                           int64_t ld_save, void* ws, size_t ws_bytes, void* stream) {
    ProjectArgs Q = {};
    int status = check_pair(gate, up, &Q.P, &Q.pair.up);
    if (status != WINDQ_OK) return status;
    status = check_tokens(X, Q.P.cols, true);
    if (status != WINDQ_OK) return status;
    if (act < WINDQ_SILU || act > WINDQ_GELU_TANH || (G == nullptr) != (U == nullptr)) return WINDQ_EINVAL;
    const size_t eb = X->dtype == WINDQ_F32 ? 4 : 2;
    if (!sizes_fit(X->rows, Q.P.rows, Q.P.cols, 0, 0)) return WINDQ_ESHAPE;
    if (ld_h < Q.P.rows || ld_h > (int64_t)1 << 31) return WINDQ_ESHAPE;
    if (G != nullptr && (ld_save < Q.P.rows || ld_save > (int64_t)1 << 31)) return WINDQ_ESHAPE;
    if (X->rows == 0) return WINDQ_OK;
    if (X->rows * Q.P.rows > (int64_t)0x7fffffff) return WINDQ_ESHAPE;
    if (H == nullptr || !aligned(H, eb) || !aligned(G, eb) || !aligned(U, eb)) return WINDQ_EINVAL;
    const GatedWs at = gated_ws(X->dtype, X->rows, Q.P.rows, Q.P.cols, Q.P.G);
    if (ws == nullptr || ws_bytes < at.total) return WINDQ_EWORKSPACE;
    if (!aligned(ws, 256)) return WINDQ_EINVAL;
    Q.X = static_cast<const uint16_t*>(X->data);
    Q.ldx = X->ld;
    Q.raw = X->data;
    Q.ld_raw = X->ld;
    Q.T = X->rows;
    Q.Y = H;
    Q.ldy = ld_h;
    Q.pair.act = act;
    Q.pair.G = G;
    Q.pair.U = U;
    Q.pair.ld_save = ld_save;
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* w = static_cast<char*>(ws);
    return X->dtype == WINDQ_F32 ? gated_all<float>(Q, X, w, at, st) : gated_all<uint16_t>(Q, X, w, at, st);
}

extern "C" int windq_gated_grad(const windq_packed* gate, const windq_packed* up, const windq_mat* dH, const void* G, const void* U, int64_t ld_save, int32_t act,
                                void* dX, int64_t ld_dx, void* dG, void* dU, int64_t ld_d, void* ws, size_t ws_bytes, void* stream) {
    SlopeArgs S = {};
    int status = check_pair(gate, up, &S.P[0], &S.P[1]);
    if (status != WINDQ_OK) return status;
    const int64_t rows = S.P[0].rows, cols = S.P[0].cols;
    status = check_tokens(dH, rows, false);
    if (status != WINDQ_OK) return status;
    const int64_t T = dH->rows;
    if (act < WINDQ_SILU || act > WINDQ_GELU_TANH || (dG == nullptr) != (dU == nullptr) || (dX == nullptr && dG == nullptr && T > 0)) return WINDQ_EINVAL;
    if (!sizes_fit(T, rows, cols, 0, 0) || !grad_sizes_fit(T, rows, cols) || rows > ((int64_t)1 << 30) - 512) return WINDQ_ESHAPE;
    if (ld_save < rows || ld_save > (int64_t)1 << 31) return WINDQ_ESHAPE;
    if (dX != nullptr && (ld_dx < cols || ld_dx > (int64_t)1 << 31)) return WINDQ_ESHAPE;
    if (dG != nullptr && (ld_d < rows || ld_d > (int64_t)1 << 31)) return WINDQ_ESHAPE;
    if (T == 0) return WINDQ_OK;
    const size_t eb = dH->dtype == WINDQ_F32 ? 4 : 2;
    if (G == nullptr || U == nullptr || !aligned(G, eb) || !aligned(U, eb) || !aligned(dX, eb) || !aligned(dG, eb) || !aligned(dU, eb)) return WINDQ_EINVAL;
    const GatedGradWs at = gated_grad_ws(dH->dtype, T, rows, cols, S.P[0].G);
    if (dX != nullptr) {
        if (ws == nullptr || ws_bytes < at.total) return WINDQ_EWORKSPACE;
        if (!aligned(ws, 256)) return WINDQ_EINVAL;
    }
    S.dH = dH->data;
    S.G = G;
    S.U = U;
    S.ld_dh = dH->ld;
    S.ld_save = ld_save;
    S.T = T;
    S.rows = rows;
    S.act = act;
    S.dG = dG;
    S.dU = dU;
    S.ld_d = ld_d;
    S.wide = dH->ld % 8 == 0 && ld_save % 8 == 0 && (dG == nullptr || ld_d % 8 == 0) && aligned(dH->data, 16) && aligned(G, 16) && aligned(U, 16) && aligned(dG, 16) && aligned(dU, 16);
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* w = static_cast<char*>(ws);
    return dH->dtype == WINDQ_F32 ? gated_grad_all<float>(S, dX, ld_dx, w, at, st) : gated_grad_all<uint16_t>(S, dX, ld_dx, w, at, st);
}
