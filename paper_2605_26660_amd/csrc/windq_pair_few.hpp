// windq_gated for a few tokens of bfloat16, or for fp32 ones: 16 rows of both matrices by 16 tokens a workgroup, the k-blocks shared by its wavefronts, half of them the gate's.
//
// Bound by unpacking and waits, not by the codes (28 MB at 2 bits for a pair of 11008 x 4096).  Tokens are the M side of 16x16x32 instructions and rows the N
// side, so that a lane has one row, with one scale and one offset, and a quarter of a k-block's columns side by side: its codes are one load of 4 to 32 bytes,
// straight to registers, and nothing but trits' table and the totals goes through LDS.  Few registers leave room for five or six wavefronts a SIMD, which
// wait for each other's loads; treatments and places of codes are looked up for all of a wavefront's k-blocks at once, ahead.
//   11008 x 4096 at 2 bits, 1 token 18.4 us, 8 tokens 23.9, 16 tokens 30.6, where 32 rows a workgroup (32x32x16 instructions, codes through LDS, one workgroup a CU: two
// rounds of them) take 35.9, 38.7 and 44.4; a k-block's codes asked for ahead of the one before: 22.3.
// fp32, 1000 x 1056, 77 tokens 27 us (by the general kernel 51), 1024 x 4096, 16 tokens 42 (100).
#pragma once

#include "windq_dx.hpp"
#include "windq_project_few.hpp"

namespace windq {

constexpr int PR_ROWS = 16;
constexpr int64_t PAIR_FEW = 16;                             // tokens of an instruction; at all of them ahead of the kernel for more

inline bool pair_fits(const PackArgs& P) {
    return P.mask == nullptr && P.rows % 8 == 0 && (P.R_u == P.rows || P.R_u % PR_ROWS == 0) && (P.G % 128 == 0 || P.G == 96 || P.G == 64);
}

#ifdef __HIPCC__

// O octets of a row (columns side by side) as f, from their first byte, in bfloat16 or (HALF) in half precision; r: trits ahead of them.
template <int O, int BITS, bool HALF = false>
__device__ __forceinline__ void pair_fields(const uint8_t* __restrict__ p, uint4 (&w)[O]) {
    uint32_t v[2 * O + 1] = {};
#pragma unroll
    for (int k = 0; k + 4 <= O * BITS; k += 4) __builtin_memcpy(&v[k >> 2], p + k, 4);
    if constexpr (O * BITS % 4 != 0) {
        uint8_t rest[4] = {};
#pragma unroll
        for (int k = 0; k < O * BITS % 4; ++k) rest[k] = p[O * BITS / 4 * 4 + k];
        v[O * BITS / 4] = (uint32_t)rest[0] | (uint32_t)rest[1] << 8 | (uint32_t)rest[2] << 16;
    }
#pragma unroll
    for (int s = 0; s < O; ++s) {
        constexpr int STEP = BITS * 8;
        const int at = s * STEP;
        if constexpr (BITS == 1) w[s] = HALF ? half_fields1((v[0] >> at) & 0xffu) : fields1((v[0] >> at) & 0xffu);
        else if constexpr (BITS == 2) w[s] = HALF ? half_fields2((v[at >> 5] >> (at & 31)) & 0xffffu) : fields2((v[at >> 5] >> (at & 31)) & 0xffffu);
        else if constexpr (BITS == 3) {
            const uint32_t q = (at & 31) <= 8 ? (v[at >> 5] >> (at & 31)) & 0xffffffu : __builtin_amdgcn_alignbit(v[(at >> 5) + 1], v[at >> 5], at & 31) & 0xffffffu;
            w[s] = HALF ? half_fields3(q) : fields3(q);
        } else if constexpr (BITS == 4) w[s] = HALF ? half_fields4(v[s]) : fields4(v[s]);
        else w[s] = HALF ? half_fields8(v[2 * s], v[2 * s + 1]) : fields8(v[2 * s], v[2 * s + 1]);
    }
}

template <int O, bool HALF = false>
__device__ __forceinline__ void pair_trits(const uint8_t* __restrict__ p, uint32_t r, const uint16_t* __restrict__ trits_of, uint4 (&w)[O]) {
    uint32_t b[2], t[8], v[3];
    __builtin_memcpy(b, p, 8);
#pragma unroll
    for (int k = 0; k < 8; ++k) t[k] = trits_of[(b[k >> 2] >> (8 * (k & 3))) & 0xffu];
    // 80 bits, two a trit
    v[0] = t[0] | t[1] << 10 | t[2] << 20 | t[3] << 30;
    v[1] = t[3] >> 2 | t[4] << 8 | t[5] << 18 | t[6] << 28;
    v[2] = t[6] >> 4 | t[7] << 6;
    if (O == 2 && r >= 16) {                                // r is below 16 for wider k-blocks
        v[0] = v[1];
        v[1] = v[2];
        r -= 16;
    }
    v[0] = __builtin_amdgcn_alignbit(v[1], v[0], 2 * r);
    if (O > 2) v[1] = __builtin_amdgcn_alignbit(v[2], v[1], 2 * r);
#pragma unroll
    for (int s = 0; s < O; ++s) {
        const uint32_t q = (s & 1) != 0 ? v[s >> 1] >> 16 : v[s >> 1] & 0xffffu;
        w[s] = HALF ? half_fields2(q) : fields2(q);
    }
}

// fp32 tokens are three planes, their codes centred.
template <typename YT, int O, int WAVES>
__global__ __launch_bounds__(WAVES * 64, sizeof(YT) == 4 ? 4 : 6) void pair_few_kernel(const FewArgs Q) {
    constexpr int NP = sizeof(YT) == 4 ? 3 : 1;
    constexpr int EACH = WAVES / 2, COLS = 32 * O;          // wavefronts of a matrix; columns of a k-block
    __shared__ float red[WAVES][4][64];
    __shared__ uint16_t trits_of[256];
    for (int i = threadIdx.x; i < 256; i += WAVES * 64) trits_of[i] = (uint16_t)trit_fields(i);
    __syncthreads();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, sub = lane & 15, q = lane >> 4;
    const int matrix = wave / EACH, turn = wave - matrix * EACH;
    const PackArgs& P = matrix == 1 ? Q.pair.up : Q.P;
    const uint32_t R_u = (uint32_t)P.R_u, block = Q.first + blockIdx.x, tb = block / Q.row_blocks, row0 = (block - tb * Q.row_blocks) * PR_ROWS, rb = row0 / R_u, lrow0 = row0 - rb * R_u;
    const int32_t rows_left = R_u - lrow0 < PR_ROWS ? (int32_t)(R_u - lrow0) : PR_ROWS;
    const uint32_t lr = (uint32_t)(sub < rows_left ? sub : rows_left - 1);
    const int32_t per_chunk = P.G / COLS;
    const int64_t unit0 = (int64_t)rb * P.n_chunks;
    const uint32_t one = 0x3f803f80u;
    const bf16x8 ones = as_bf16x8(make_uint4(one, one, one, one));
    const int64_t t0 = (int64_t)tb * 16;
    const int32_t tokens = Q.T - t0 < 16 ? (int32_t)(Q.T - t0) : 16;
    const uint16_t* const x0 = Q.X + (t0 + (sub < tokens ? sub : tokens - 1)) * Q.ldx + q * (8 * O);

    f32x4 tot = {};
    for (int32_t from = turn; from < Q.n_kb; from += 64 * EACH) {
        // of the wavefront's next 64 k-blocks, a lane each: the chunk, and where the unit's rows start, with bytes of a row and treatment above
        const int32_t mine = from + lane * EACH;
        uint64_t word = 0;
        uint32_t chunk = 0;
        if (mine < Q.n_kb) {
            chunk = (uint32_t)mine / (uint32_t)per_chunk;
            int64_t base;
            const int a = pk_action(P, unit0 + chunk, base);
            const int64_t bytes = pk_bytes_per_group(a, P.G);
            if (a != 0) word = (uint64_t)(base + lrow0 * bytes) | (uint64_t)bytes << 48 | (uint64_t)a << 61;      // tensors are no longer than 2^42 bytes
        }
        const int32_t count = (Q.n_kb - from + EACH - 1) / EACH < 64 ? (Q.n_kb - from + EACH - 1) / EACH : 64;
        for (int32_t it = 0; it < count; ++it) {
            const int32_t kb = from + it * EACH, j = __builtin_amdgcn_readlane((int)chunk, it), c = kb - j * per_chunk;
            const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(word >> 32), it), bpg = hi >> 16 & 0x1fffu;
            const int kind = (int)(hi >> 29);
            const uint8_t* const codes = P.codes + ((uint64_t)(hi & 0xffffu) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)word, it));
            const int64_t g = (unit0 + j) * R_u + lrow0;
            const float scale = (P.scale + g)[lr], offset = (P.offset + g)[lr];
            uint4 x[NP][O], w[O];
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int s = 0; s < O; ++s) x[p][s] = reinterpret_cast<const uint4*>(x0 + p * Q.plane + (int64_t)kb * COLS)[s];
            const uint32_t first = (uint32_t)c * COLS + q * (8 * O), row = lr * bpg;
            switch (kind) {
                case 1: pair_fields<O, 8>(codes + (row + first), w); break;
                case 2: pair_fields<O, 4>(codes + (row + (first >> 1)), w); break;
                case 3: pair_fields<O, 3>(codes + (row + (first >> 3) * 3), w); break;
                case 4: pair_fields<O, 2>(codes + (row + (first >> 2)), w); break;
                case 5: {
                    const uint32_t k = first / 5u, at = k < bpg - 8u ? k : bpg - 8u;      // eight bytes within the row
                    pair_trits<O>(codes + (row + at), first - at * 5u, trits_of, w);
                    break;
                }
                case 6: pair_fields<O, 1>(codes + (row + (first >> 3)), w); break;
                default: {
                    const uint16_t* const from = static_cast<const uint16_t*>(P.W) + (int64_t)(row0 + lr) * P.ld + (int64_t)kb * COLS + q * (8 * O);
#pragma unroll
                    for (int s = 0; s < O; ++s) w[s] = P.w_f32 != 0 ? make_uint4(0u, 0u, 0u, 0u) : reinterpret_cast<const uint4*>(from)[s];
                }
            }
            f32x4 acc = {}, sums = {};
#pragma unroll
            for (int s = 0; s < O; ++s) {
                if (NP == 3 && kind != 0) w[s] = centred(w[s], pk_centre(kind));
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) {
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(x[p][s]), as_bf16x8(w[s]), acc, 0, 0, 0);
                    sums = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(x[p][s]), ones, sums, 0, 0, 0);
                }
            }
            if (kind == 0 && P.w_f32 != 0) {
#pragma unroll 1
                for (int i = 0; i < 3 * O; ++i) {           // rare: three terms of an octet, x once more from where it lies
                    const int term = i / O, s = i - term * O;
                    const uint4 v = skip_octet(P, row0 + lr, (int64_t)kb * COLS + q * (8 * O) + s * 8, term);
#pragma unroll
                    for (int p = 0; p < NP; ++p)
                        if (NP == 1 || p + term < 3)
                            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(reinterpret_cast<const uint4*>(x0 + p * Q.plane + (int64_t)kb * COLS)[s]), as_bf16x8(v), acc, 0, 0, 0);
                }
            }
            float alpha, beta;
            pk_affine(kind, scale, offset, NP == 3, alpha, beta);
#pragma unroll
            for (int i = 0; i < 4; ++i) tot[i] = fmaf(alpha, acc[i], fmaf(beta, sums[i], tot[i]));
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) red[wave][i][lane] = tot[i];
    __syncthreads();
    for (int e = threadIdx.x; e < PR_ROWS * tokens; e += WAVES * 64) {
        const int r = e & 15, n = e >> 4, at = (n >> 2) * 16 + r;      // neighbouring lanes: neighbouring rows of a token
        if (r >= rows_left) continue;
        float v = 0.0f, up = 0.0f;
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            v += red[k][n & 3][at];
            up += red[EACH + k][n & 3][at];
        }
        const int64_t row = (int64_t)row0 + r, t = t0 + n;
        const YT* const raw = static_cast<const YT*>(Q.raw) + t * Q.ld_raw;
        if (!isfinite(v)) v = (float)pk_slow_dot(Q.P, row, raw);
        if (!isfinite(up)) up = (float)pk_slow_dot(Q.pair.up, row, raw);
        store_y(reinterpret_cast<YT*>(Q.Y) + t * Q.ldy + row, pair_result<YT>(Q.pair, t, row, v, up));
    }
}

template <typename YT, int O>
int launch_pair_few(FewArgs Q, hipStream_t st) {
    Q.row_blocks = (uint32_t)tokens_in(Q.P.rows, PR_ROWS);
    const int64_t wgs = Q.row_blocks * tokens_in(Q.T, 16);
    return launch_pieces(wgs, wgs > 512 ? 512 : 1024, [&](int64_t first, dim3 g) {
        Q.first = (uint32_t)first;
        // eight wavefronts where there are two workgroups a CU and more, so that all of them run at once
        if (wgs > 512) pair_few_kernel<YT, O, 8><<<g, dim3(512), 0, st>>>(Q);
        else pair_few_kernel<YT, O, 16><<<g, dim3(1024), 0, st>>>(Q);
    });
}

// Chunks of whole k-blocks (given by their sixteens of columns).
template <typename YT>
int launch_pair_few(FewArgs F, hipStream_t st) {
    const int steps = F.P.G % 128 == 0 ? 8 : F.P.G / 16;
    F.n_kb = (int32_t)(F.P.cols / (16 * steps));
    return steps == 8 ? launch_pair_few<YT, 4>(F, st) : (steps == 6 ? launch_pair_few<YT, 3>(F, st) : launch_pair_few<YT, 2>(F, st));
}

#endif  // __HIPCC__

}  // namespace windq
