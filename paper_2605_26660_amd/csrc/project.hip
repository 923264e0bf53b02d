// windq_project: a batch of tokens through a packed matrix, each with the low-rank adapter of its own request beside it.
//   Y[t] = w_hat x_t + alpha_k B_k h_t,   h_t = A_k x_t,   k = adapter_of[t]
#include <math.h>

#include "windq_project_few.hpp"

namespace windq {

// ------------------------------------------------------------------------------------------------ fp32 activations
// X in fp32 enters the products as three planes of bfloat16 that add up to it.
__global__ __launch_bounds__(256) void planes_kernel(const float* __restrict__ X, int64_t ldx, int64_t T, int32_t cols, uint16_t* __restrict__ planes) {
    const int64_t octets = cols >> 3;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= T * octets) return;
    const int64_t t = i / octets, c = (i - t * octets) * 8;
    uint32_t v[3][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) split3(X[t * ldx + c + j], v[0][j], v[1][j], v[2][j]);
#pragma unroll
    for (int k = 0; k < 3; ++k)
        *reinterpret_cast<uint4*>(planes + (k * T + t) * cols + c) =
            make_uint4(v[k][0] | v[k][1] << 16, v[k][2] | v[k][3] << 16, v[k][4] | v[k][5] << 16, v[k][6] | v[k][7] << 16);
}

// ------------------------------------------------------------------------------------------------ the product, any shape
// A workgroup has 16 rows and 16 NT tokens; its eight wavefronts share the chunks among them and add up through LDS.  A
// wavefront's rows are the M side of 16x16x32 matrix instructions: lane l has row l mod 16 and, of every chunk, the octets
// of its quarter l / 16.  Which columns the four quarters pair up is free as long as X's operand does the same, so a lane's octets lie next to
// each other and its codes are contiguous bytes.  sum_c x comes from the same instructions with ones for weights (under a mask: ones
// where the weight is kept).
constexpr int PJ_WAVES = 8;
constexpr int64_t PROJECT_FEW = 64;                       // tokens up to which this kernel, or that for few tokens, is the faster one

struct ProjectArgs {
    PackArgs P;
    const uint16_t* X;         // bfloat16, or the first of three planes
    int64_t ldx, plane;        // elements between tokens, and between planes
    const void* raw;           // the caller's X
    int64_t ld_raw;
    int64_t T;
    void* Y;
    int64_t ldy;
    const float* h;            // or null: no adapters
    AdapterArgs A;
    int64_t first;             // of the workgroups of this launch
};

template <typename YT>
__device__ __forceinline__ void store_y(YT* __restrict__ p, float v) {
    if constexpr (sizeof(YT) == 4) *p = v;
    else *p = (uint16_t)f32_to_bf16_bits(v);
}

template <typename YT, int NT, bool MASK>
__global__ __launch_bounds__(PJ_WAVES * 64) void project_kernel(const ProjectArgs Q) {
    constexpr int NP = sizeof(YT) == 4 ? 3 : 1;
    __shared__ float red[PJ_WAVES][NT * 4][64];
    __shared__ uint16_t trits_of[256];
    if (threadIdx.x < 256) trits_of[threadIdx.x] = (uint16_t)trit_fields(threadIdx.x);
    __syncthreads();
    const PackArgs& P = Q.P;
    const int32_t G = P.G, O = G >> 3, S = (O + 3) >> 2;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, sub = lane & 15, q = lane >> 4;
    const int64_t row_blocks = (P.rows + 15) / 16;
    const int64_t block = Q.first + blockIdx.x, tb = block / row_blocks;
    const int64_t row0 = (block - tb * row_blocks) * 16, t0 = tb * (NT * 16);

    const uint16_t* xp[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int64_t t = t0 + n * 16 + sub;
        xp[n] = Q.X + (t < Q.T ? t : Q.T - 1) * Q.ldx;
    }
    const int64_t row = row0 + sub < P.rows ? row0 + sub : P.rows - 1;        // past the last one: computed for nothing, stored by nobody
    const int64_t rb = row / P.R_u, lrow = row - rb * P.R_u;
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    const uint32_t one = 0x3f803f80u;
    const uint4 ones = make_uint4(one, one, one, one);

    f32x4 tot[NT] = {};
    for (int32_t j = wave; j < P.n_chunks; j += PJ_WAVES) {
        const int64_t u = rb * P.n_chunks + j, g = u * P.R_u + lrow;
        int64_t base;
        const int act = pk_action(P, u, base);
        const uint8_t* const codes = P.codes + base + lrow * pk_bytes_per_group(act, G);
        float alpha, beta;
        pk_affine(act, P.scale[g], P.offset[g], NP == 3, alpha, beta);
        const bool wide = act == 0 && P.w_f32 != 0;         // fp32 skip weights
        f32x4 acc[NT] = {}, xs[NT] = {};
        for (int32_t s = 0; s < S; ++s) {
            const int32_t o = q * S + s;
            const bool valid = o < O;
            const int64_t col = (int64_t)j * G + o * 8;
            bf16x8 b[NP][NT];
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int n = 0; n < NT; ++n) b[p][n] = as_bf16x8(valid ? *reinterpret_cast<const uint4*>(xp[n] + p * Q.plane + col) : none);
            uint4 w = none, k = ones;
            if (valid) {
                w = act == 0 ? skip_octet(P, row, col, 0) : octet_fields(act, codes, o, trits_of);
                if (NP == 3 && act != 0) w = centred(w, pk_centre(act));
                if (MASK && act != 0) {
                    k = keep_words(P.mask[row * P.mask_ld + (col >> 3)]);
                    w = and4(w, k);
                    k = and4(k, ones);
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) {
                    acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(w), b[p][n], acc[n], 0, 0, 0);
                    xs[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(k), b[p][n], xs[n], 0, 0, 0);
                }
            if (__any(wide)) {
                for (int term = 1; term < 3; ++term) {
                    const uint4 more = valid && act == 0 ? skip_octet(P, row, col, term) : none;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int p = 0; p < NP; ++p)
                            if (p + term < 3) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(more), b[p][n], acc[n], 0, 0, 0);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float al = __shfl(alpha, 4 * q + i, 64), be = __shfl(beta, 4 * q + i, 64);
#pragma unroll
            for (int n = 0; n < NT; ++n) tot[n][i] = fmaf(al, acc[n][i], fmaf(be, xs[n][i], tot[n][i]));
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) red[wave][n * 4 + i][lane] = tot[n][i];
    __syncthreads();
    YT* __restrict__ const Y = static_cast<YT*>(Q.Y);
    for (int e = threadIdx.x; e < NT * 256; e += PJ_WAVES * 64) {
        // row by row within a token, so that neighbouring lanes write neighbouring rows
        const int r = e & 15, n = e >> 4;
        const int64_t y = row0 + r, t = t0 + n;
        if (y >= P.rows || t >= Q.T) continue;
        const int slot = (n >> 4) * 4 + (r & 3), at = (r >> 2) * 16 + (n & 15);
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < PJ_WAVES; ++w) v += red[w][slot][at];
        if (!isfinite(v)) v = (float)pk_slow_dot(P, y, static_cast<const YT*>(Q.raw) + t * Q.ld_raw);
        if (Q.h != nullptr) v += expand_one<YT>(Q.A, Q.h, t, y, P.rows);
        store_y(Y + t * Q.ldy + y, v);
    }
}

template <typename YT, int NT, bool MASK>
int launch_project(ProjectArgs Q, hipStream_t st) {
    return launch_pieces(tokens_in(Q.P.rows, 16) * tokens_in(Q.T, NT * 16), PJ_WAVES * 64, [&](int64_t first, dim3 g) {
        Q.first = first;
        project_kernel<YT, NT, MASK><<<g, dim3(PJ_WAVES * 64), 0, st>>>(Q);
    });
}

// Sixteen tokens a workgroup while that leaves two workgroups a CU at most: their time is latency.  fp32, 1000 x 1056: 77 tokens (315 of them) 35 us,
// 58 with 64 tokens each; 512 x 512, 64 tokens (128) 12 and 29; bfloat16, 1024 x 1120, 64 tokens (256) 9 and 21.  Else 32, so that a weight
// is unpacked half as often: bfloat16, 4096 x 4000, 2000 tokens 1863 us, 2041 with 16 each and 1895 with 64.
template <typename YT, bool MASK>
int launch_project_any(const ProjectArgs& Q, hipStream_t st) {
    if (tokens_in(Q.P.rows, 16) * tokens_in(Q.T, 16) <= 512) return launch_project<YT, 1, MASK>(Q, st);
    return launch_project<YT, 2, MASK>(Q, st);
}

int check_packed(const windq_packed* P, PackArgs* A) {
    if (P == nullptr) return WINDQ_EINVAL;
    Geometry g;
    const int status = make_geometry(P->W, P->chunk_w, P->unit_rows, &g);
    if (status != WINDQ_OK) return status;
    if (P->action == nullptr || P->code_off == nullptr || P->scale == nullptr || P->offset == nullptr) return WINDQ_EINVAL;
    if (P->codes == nullptr && P->codes_bytes != 0) return WINDQ_EINVAL;     // no codes: skip units alone
    if (!aligned(P->code_off, 8) || !aligned(P->codes, 16) || !aligned(P->scale, 4) || !aligned(P->offset, 4)) return WINDQ_EINVAL;
    A->W = P->W->data;
    A->ld = P->W->ld;
    A->w_f32 = P->W->dtype == WINDQ_F32;
    A->mask = P->mask;
    A->mask_ld = g.cols / 8;
    A->action = P->action;
    A->code_off = P->code_off;
    A->codes = P->codes;
    A->codes_bytes = (int64_t)P->codes_bytes;
    A->scale = P->scale;
    A->offset = P->offset;
    A->rows = g.rows;
    A->cols = g.cols;
    A->R_u = g.R_u;
    A->G = g.chunk_w;
    A->n_chunks = (int32_t)g.n_chunks;
    return WINDQ_OK;
}

int check_adapters(const windq_adapters* ad, const int32_t* adapter_of, int32_t dtype, AdapterArgs* A) {
    if (ad->a == nullptr || ad->b == nullptr || adapter_of == nullptr) return WINDQ_EINVAL;
    if (ad->dtype != WINDQ_F32 && ad->dtype != WINDQ_BF16) return WINDQ_EDTYPE;
    if (ad->dtype != dtype) return WINDQ_EDTYPE;
    if (ad->n < 1 || ad->n > WINDQ_MAX_ADAPTERS || ad->max_rank < 8 || ad->max_rank > WINDQ_MAX_RANK || ad->max_rank % 8 != 0) return WINDQ_ESHAPE;
    if (!aligned(ad->a, 16) || !aligned(ad->b, 16) || !aligned(ad->alpha, 4) || !aligned(ad->rank, 4) || !aligned(adapter_of, 4)) return WINDQ_EINVAL;
    A->a = ad->a;
    A->b = ad->b;
    A->alpha = ad->alpha;
    A->rank = ad->rank;
    A->of = adapter_of;
    A->n = ad->n;
    A->max_rank = ad->max_rank;
    return WINDQ_OK;
}

// Activations or their gradients: [tokens][width], no tokens is fine.  `vector`: read eight at a time.
int check_tokens(const windq_mat* M, int64_t width, bool vector) {
    if (M == nullptr) return WINDQ_EINVAL;
    if (M->dtype != WINDQ_F32 && M->dtype != WINDQ_BF16) return WINDQ_EDTYPE;
    if (M->rows < 0 || M->cols != width || M->ld < M->cols || M->rows > ((int64_t)1 << 31) - 1 || M->ld > (int64_t)1 << 31) return WINDQ_ESHAPE;
    if (vector && M->ld % 8 != 0) return WINDQ_ESHAPE;
    if (M->rows == 0) return WINDQ_OK;
    if (M->data == nullptr || !aligned(M->data, vector ? 16 : (M->dtype == WINDQ_F32 ? 4 : 2))) return WINDQ_EINVAL;
    return WINDQ_OK;
}

size_t grad_ws_bytes(int32_t dtype, int64_t T, int64_t rows, int64_t cols, int32_t n, int32_t max_rank);

// Offsets of a workspace's parts.  They are those of the shape alone, so that fewer tokens, or rows in other units, never need more.
struct ProjectWs {
    size_t planes, h, frag, few_xs, place, owner, first, count, part, fields, unit, xs, beta, alpha, total;
};

ProjectWs project_ws(int32_t dtype, int64_t T, int64_t rows, int64_t cols, int32_t G, int32_t n, int32_t max_rank) {
    ProjectWs w;
    size_t at = 0;
    auto take = [&at](size_t bytes) {
        const size_t here = at;
        at += round_up(bytes, 256);
        return here;
    };
    w.planes = take(dtype == WINDQ_F32 ? (size_t)(3 * T * cols) * 2 : 0);
    w.h = take((size_t)(T * max_rank) * 4);
    const bool few = dtype == WINDQ_BF16;                   // fewer tokens than asked for fit too
    const int64_t few_tokens = T < few_most(rows, cols, G) ? tokens_in(T, 64) * 64 : few_most(rows, cols, G);
    w.frag = take(few ? (size_t)cols * (size_t)few_tokens * 2 : 0);
    w.few_xs = take(few ? (size_t)(cols / 64 + 1) * (size_t)few_tokens * 4 : 0);
    const bool grouped = n > 0 && dtype == WINDQ_BF16 && T > SHRINK_FEW;
    const int64_t slots = group_slots(T, n);
    w.place = take(grouped ? (size_t)slots * GROUP * 4 : 0);
    w.owner = take(grouped ? (size_t)slots * 4 : 0);
    w.first = take(grouped ? (size_t)n * 4 : 0);
    w.count = take(grouped ? (size_t)n * 4 : 0);
    w.part = take(grouped ? shrink_floats(slots, cols, max_rank) * 4 : 0);
    const bool many = T > PROJECT_FEW;
    w.fields = take(many ? (size_t)(rows * cols) / (G == 128 || G == 96 || G == 64 ? 2 : 1) : 0);
    w.unit = take(many ? (size_t)((rows + PT_STRIP - 1) / PT_STRIP) * (size_t)(cols / 64) * sizeof(KbWord) : 0);
    w.xs = take(many ? (size_t)(cols / 64) * (size_t)T * 16 : 0);
    w.beta = take(many ? (size_t)(cols / 64) * (size_t)rows * 16 : 0);
    w.alpha = take(many ? (size_t)(cols / G) * (size_t)rows * 4 : 0);
    w.total = at == 0 ? 256 : at;
    return w;
}

// Tiles for many tokens (windq_project_tiles.hpp).
template <typename XT, int S>
int launch_tiles(const ProjectArgs& Q, char* ws, const ProjectWs& at, hipStream_t st) {
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
    A.h = Q.h;
    A.A = Q.A;
    A.fields = reinterpret_cast<uint8_t*>(ws + at.fields);
    A.unit = reinterpret_cast<KbWord*>(ws + at.unit);
    A.xs = reinterpret_cast<uint4*>(ws + at.xs);
    A.beta = reinterpret_cast<uint4*>(ws + at.beta);
    A.alpha = reinterpret_cast<float*>(ws + at.alpha);
    A.unit_fields = Q.P.R_u * Q.P.G / (tile_natural(Q.P.G, S) ? 2 : 1);
    A.n_kb = (int32_t)(Q.P.cols / (16 * S));
    A.row_blocks = (uint32_t)((Q.P.rows + PT_ROWS - 1) / PT_ROWS);
    const int64_t strips = (Q.P.rows / Q.P.R_u) * Q.P.n_chunks * ((Q.P.R_u + PT_STRIP - 1) / PT_STRIP);
    const int64_t wgs = strips + tokens_in(A.n_kb * Q.T, PT_SUMS);
    const int64_t tiles = (int64_t)A.row_blocks * ((Q.T + PT_TOKENS - 1) / PT_TOKENS);
    // tiles are no more than 2^31 / (64 x 128) and two sides' edges: one launch holds them
    const int status = launch_pieces(wgs, 256, [&](int64_t first, dim3 g) { tiles_prepare_kernel<XT, S><<<g, dim3(256), 0, st>>>(A, strips, first); });
    if (status != WINDQ_OK) return status;
    project_tiles_kernel<XT, S><<<dim3((uint32_t)tiles), dim3(PT_THREADS), 0, st>>>(A);
    return hipGetLastError() == hipSuccess ? WINDQ_OK : WINDQ_EHIP;
}

template <typename XT>
int project_all(ProjectArgs& Q, const windq_mat* X, const windq_adapters* ad, float* h, char* ws, const ProjectWs& at, hipStream_t st) {
    const int64_t T = Q.T;
    if constexpr (sizeof(XT) == 4) {
        uint16_t* planes = reinterpret_cast<uint16_t*>(ws + at.planes);
        const int64_t pieces = T * (Q.P.cols / 8);
        if (!fits_launch((pieces + 255) / 256, 256)) return WINDQ_ESHAPE;
        planes_kernel<<<dim3((uint32_t)((pieces + 255) / 256)), dim3(256), 0, st>>>(static_cast<const float*>(X->data), X->ld, T, (int32_t)Q.P.cols, planes);
        if (hipGetLastError() != hipSuccess) return WINDQ_EHIP;
        Q.X = planes;
        Q.ldx = Q.P.cols;
        Q.plane = T * Q.P.cols;
    }
    // Few tokens' h is formed by the kernel that lays X out, a wavefront a rank.
    const bool few = sizeof(XT) == 2 && few_fits(Q.P, T), own_h = few && T <= FEW_OWN_H;
    float* const ht = ad == nullptr ? nullptr : (h != nullptr ? h : reinterpret_cast<float*>(ws + at.h));
    if (ad != nullptr && !own_h) {
        bool grouped = false;
        if constexpr (sizeof(XT) == 2) {
            grouped = T > SHRINK_FEW;
            if (grouped) {
                GroupArgs G = {Q.A.of, T, Q.A.n, group_slots(T, Q.A.n), reinterpret_cast<int32_t*>(ws + at.place), reinterpret_cast<int32_t*>(ws + at.owner),
                               reinterpret_cast<int32_t*>(ws + at.first), reinterpret_cast<int32_t*>(ws + at.count)};
                ShrinkArgs S = {X->data, X->ld, Q.A.a, Q.P.cols, (int32_t)Q.P.cols, shrink_splits(G.slots, Q.P.cols), G.slots, G.place, G.owner, Q.A,
                                reinterpret_cast<float*>(ws + at.part)};
                JoinArgs J = {S.part, S.splits, G.slots, G.place, G.owner, T, Q.A, false, ht, nullptr, nullptr};
                int status = launch_group(G, st);
                if (status == WINDQ_OK) status = launch_shrink(S, nullptr, st);
                if (status == WINDQ_OK) status = launch_join(J, nullptr, st);
                if (status != WINDQ_OK) return status;
            }
        }
        if (!grouped) {
            const int status = launch_shrink_token(static_cast<const XT*>(X->data), X->ld, T, (int32_t)Q.P.cols, Q.A, false, ht, st);
            if (status != WINDQ_OK) return status;
        }
    }
    Q.h = ht;
    if constexpr (sizeof(XT) == 2) {
        if (few) {
            FewArgs F = {Q.P, Q.X, Q.ldx, T, static_cast<uint16_t*>(Q.Y), Q.ldy, ht, Q.A, 0, reinterpret_cast<uint4*>(ws + at.frag), reinterpret_cast<float*>(ws + at.few_xs), 0, 0, 0};
            const int steps = Q.P.G % 128 == 0 ? 8 : Q.P.G / 16;
            F.n_kb = (int32_t)(Q.P.cols / (16 * steps));
            float* const form = own_h ? ht : nullptr;
            return steps == 8 ? launch_few<8>(F, form, st) : (steps == 6 ? launch_few<6>(F, form, st) : launch_few<4>(F, form, st));
        }
    }
    // The general kernel where its workgroups run about at once.  bfloat16, 1024 x 1024: 160 tokens (192 of them) 21 us, tiles 31; 320 tokens (320) 39
    // and 31.  fp32, 4096 x 4096: 80 tokens (512) 237 us, tiles 303; 160 tokens (768) 450 and 312.
    const int64_t general = (Q.P.rows + 15) / 16 * tokens_in(T, 64);
    const int S = Q.P.mask == nullptr && T > PROJECT_FEW && general > (sizeof(XT) == 2 ? 256 : 512) ? tile_steps(Q.P) : 0;
    if (S == 8) return launch_tiles<XT, 8>(Q, ws, at, st);
    if (S == 6) return launch_tiles<XT, 6>(Q, ws, at, st);
    if (S == 4) return launch_tiles<XT, 4>(Q, ws, at, st);
    return Q.P.mask != nullptr ? launch_project_any<XT, true>(Q, st) : launch_project_any<XT, false>(Q, st);
}

}  // namespace windq

using namespace windq;

extern "C" size_t windq_project_workspace_bytes(int32_t grad, int32_t dtype, int64_t tokens, int64_t rows, int64_t cols,
                                                int32_t chunk_w, int32_t n_adapters, int32_t max_rank) {
    if ((dtype != WINDQ_F32 && dtype != WINDQ_BF16) || tokens < 0 || rows <= 0 || cols <= 0 || chunk_w <= 0 || n_adapters < 0 || max_rank < 0) return 0;
    if (n_adapters == 0 && max_rank <= WINDQ_MAX_RANK) max_rank = 0;
    if (!sizes_fit(tokens, rows, cols, n_adapters, max_rank) || (grad != 0 && !grad_sizes_fit(tokens, rows, cols))) return 0;
    return grad != 0 ? grad_ws_bytes(dtype, tokens, rows, cols, n_adapters, max_rank) : project_ws(dtype, tokens, rows, cols, chunk_w, n_adapters, max_rank).total;
}

extern "C" int windq_project(const windq_packed* P, const windq_mat* X, const windq_adapters* adapters, const int32_t* adapter_of,
                             void* Y, int64_t ld_y, float* h, void* ws, size_t ws_bytes, void* stream) {
    ProjectArgs Q = {};
    int status = check_packed(P, &Q.P);
    if (status != WINDQ_OK) return status;
    status = check_tokens(X, Q.P.cols, true);
    if (status != WINDQ_OK) return status;
    if (adapters != nullptr) {
        static const int32_t nobody = -1;                  // no tokens: no list of theirs either
        status = check_adapters(adapters, X->rows == 0 ? &nobody : adapter_of, X->dtype, &Q.A);
        if (status != WINDQ_OK) return status;
        if (!aligned(h, 16)) return WINDQ_EINVAL;
    }
    const size_t eb = X->dtype == WINDQ_F32 ? 4 : 2;
    if (!sizes_fit(X->rows, Q.P.rows, Q.P.cols, Q.A.n, Q.A.max_rank)) return WINDQ_ESHAPE;
    if (ld_y < Q.P.rows || ld_y > (int64_t)1 << 31) return WINDQ_ESHAPE;
    if (X->rows == 0) return WINDQ_OK;
    if (X->rows * Q.P.rows > (int64_t)0x7fffffff) return WINDQ_ESHAPE;
    if (Y == nullptr || !aligned(Y, eb)) return WINDQ_EINVAL;
    const ProjectWs at = project_ws(X->dtype, X->rows, Q.P.rows, Q.P.cols, Q.P.G, Q.A.n, Q.A.max_rank);
    if (ws == nullptr || ws_bytes < at.total) return WINDQ_EWORKSPACE;
    if (!aligned(ws, 256)) return WINDQ_EINVAL;
    Q.X = static_cast<const uint16_t*>(X->data);
    Q.ldx = X->ld;
    Q.raw = X->data;
    Q.ld_raw = X->ld;
    Q.T = X->rows;
    Q.Y = Y;
    Q.ldy = ld_y;
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* w = static_cast<char*>(ws);
    return X->dtype == WINDQ_F32 ? project_all<float>(Q, X, adapters, h, w, at, st) : project_all<uint16_t>(Q, X, adapters, h, w, at, st);
}
