// windq_project: a batch of tokens through a packed matrix, each with the low-rank adapter of its own request beside it.
//   Y[t] = w_hat x_t + alpha_k B_k h_t,   h_t = A_k x_t,   k = adapter_of[t]
#include <math.h>

#include "windq_project_any.hpp"

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

int launch_planes(const float* X, int64_t ldx, int64_t T, int32_t cols, uint16_t* planes, hipStream_t st) {
    const int64_t pieces = T * (cols / 8);
    if (!fits_launch((pieces + 255) / 256, 256)) return WINDQ_ESHAPE;
    planes_kernel<<<dim3((uint32_t)((pieces + 255) / 256)), dim3(256), 0, st>>>(X, ldx, T, cols, planes);
    return hipGetLastError() == hipSuccess ? WINDQ_OK : WINDQ_EHIP;
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
        const int status = launch_planes(static_cast<const float*>(X->data), X->ld, T, (int32_t)Q.P.cols, planes, st);
        if (status != WINDQ_OK) return status;
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
            FewArgs F = {Q.P, Q.X, Q.ldx, T, static_cast<uint16_t*>(Q.Y), Q.ldy, ht, Q.A, 0, reinterpret_cast<uint4*>(ws + at.frag), reinterpret_cast<float*>(ws + at.few_xs), 0, 0, 0, 0};
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
