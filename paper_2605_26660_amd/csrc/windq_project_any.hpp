// windq_project's kernel for any shape, and windq_gated's.
#pragma once

#include "windq_project_few.hpp"

namespace windq {

// A workgroup has 16 rows and 16 NT tokens; its eight wavefronts share the chunks among them and add up through LDS.  A
// wavefront's rows are the M side of 16x16x32 matrix instructions: lane l has row l mod 16 and, of every chunk, the octets
// of its quarter l / 16.  Which columns the four quarters pair up is free as long as X's operand does the same, so a lane's octets lie next to
// each other and its codes are contiguous bytes.  sum_c x comes from the same instructions with ones for weights (under a mask: ones
// where the weight is kept).
//   Of a pair (windq_gated) half of the wavefronts has the gate's chunks, the others the up's, and what meets in LDS is both of a result's products.
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
    PairArgs pair;
};

int launch_planes(const float* X, int64_t ldx, int64_t T, int32_t cols, uint16_t* planes, hipStream_t st);

#ifdef __HIPCC__

template <typename YT, int NT, bool MASK, bool PAIR = false>
__global__ __launch_bounds__(PJ_WAVES * 64) void project_kernel(const ProjectArgs Q) {
    constexpr int NP = sizeof(YT) == 4 ? 3 : 1;
    __shared__ float red[PJ_WAVES][NT * 4][64];
    __shared__ uint16_t trits_of[256];
    if (threadIdx.x < 256) trits_of[threadIdx.x] = (uint16_t)trit_fields(threadIdx.x);
    __syncthreads();
    constexpr int EACH = PAIR ? PJ_WAVES / 2 : PJ_WAVES;   // wavefronts of a matrix
    const int matrix = PAIR ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / EACH : 0;
    const PackArgs& P = PAIR && matrix == 1 ? Q.pair.up : Q.P;
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
    for (int32_t j = wave - matrix * EACH; j < P.n_chunks; j += EACH) {
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
                if (MASK && act != 0 && (!PAIR || P.mask != nullptr)) {
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
        for (int w = 0; w < EACH; ++w) v += red[w][slot][at];
        if (!isfinite(v)) v = (float)pk_slow_dot(Q.P, y, static_cast<const YT*>(Q.raw) + t * Q.ld_raw);
        if constexpr (PAIR) {
            float up = 0.0f;
#pragma unroll
            for (int w = EACH; w < PJ_WAVES; ++w) up += red[w][slot][at];
            if (!isfinite(up)) up = (float)pk_slow_dot(Q.pair.up, y, static_cast<const YT*>(Q.raw) + t * Q.ld_raw);
            v = pair_result<YT>(Q.pair, t, y, v, up);
        } else if (Q.h != nullptr) {
            v += expand_one<YT>(Q.A, Q.h, t, y, P.rows);
        }
        store_y(Y + t * Q.ldy + y, v);
    }
}

template <typename YT, int NT, bool MASK, bool PAIR = false>
int launch_project(ProjectArgs Q, hipStream_t st) {
    return launch_pieces(tokens_in(Q.P.rows, 16) * tokens_in(Q.T, NT * 16), PJ_WAVES * 64, [&](int64_t first, dim3 g) {
        Q.first = first;
        project_kernel<YT, NT, MASK, PAIR><<<g, dim3(PJ_WAVES * 64), 0, st>>>(Q);
    });
}

// Sixteen tokens a workgroup while that leaves two workgroups a CU at most: their time is latency.  fp32, 1000 x 1056: 77 tokens (315 of them) 35 us,
// 58 with 64 tokens each; 512 x 512, 64 tokens (128) 12 and 29; bfloat16, 1024 x 1120, 64 tokens (256) 9 and 21.  Else 32, so that a weight
// is unpacked half as often: bfloat16, 4096 x 4000, 2000 tokens 1863 us, 2041 with 16 each and 1895 with 64.
template <typename YT, bool MASK, bool PAIR = false>
int launch_project_any(const ProjectArgs& Q, hipStream_t st) {
    if (tokens_in(Q.P.rows, 16) * tokens_in(Q.T, 16) <= 512) return launch_project<YT, 1, MASK, PAIR>(Q, st);
    return launch_project<YT, 2, MASK, PAIR>(Q, st);
}

#endif  // __HIPCC__

}  // namespace windq
