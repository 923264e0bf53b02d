// windq_project for few tokens of bfloat16 (up to 64, or more where rows are few): 32 rows and up to 64 tokens a workgroup, the k-blocks shared by its wavefronts.
//
// Bound by latency, not by the codes: 7 MB at 2 bits for 11008 x 4096.  So the sum is cut into as many pieces as there are k-blocks per
// wavefront, every wavefront works by itself until the end, and what it needs of a k-block is asked for at once: codes by direct
// loads to a place of its own in LDS, scales and X into registers, and the next k-block's treatment behind them.  Its 32 rows are the
// M side of 32x32x16 instructions; a lane takes half of a row's columns of a k-block, so codes are read as they lie, trits by table.
//   X is read by every workgroup, so a kernel ahead (with the adapters' first half, if there is one) lays it out in the order in which the
// lanes want it, 1 KB a load, and sums it up.  Up to FEW_DIRECT tokens it is read as it lies, and summed up by instructions with ones for weights.
//   Totals meet in LDS, in the order of the wavefronts.
//   1 token through 4096 x 4096 at 2 bits 12 us (+ 3 for h), 48 tokens of 32 adapters through 11008 x 4096 44 to 46 us (+ 5): two rounds of workgroups, waits
// are 59 % of the wavefronts' time.
#pragma once

#include "windq_project_tiles.hpp"

namespace windq {

constexpr int PF_ROWS = 32;

struct FewArgs {
    PackArgs P;
    const uint16_t* X;
    int64_t ldx, T;
    uint16_t* Y;
    int64_t ldy;
    const float* h;            // or null: no adapters
    AdapterArgs A;
    int32_t n_kb;
    uint4* frag;               // [k-blocks][fragments][S][64 lanes], or unused
    float* xs;                 // [k-blocks][xs_ld]
    int64_t xs_ld;             // tokens in 64s
    int32_t fragments;         // of 32 tokens
    uint32_t row_blocks;
};

// Up to FEW_DIRECT tokens X is read as it lies, a launch less: at 8 tokens 4096 x 4096 takes 13.7 us and 18.5 laid out, 11008 x 4096 25.7 and 31.4 (at 16
// 4096 x 4096 would still take 16.2 instead of 19.4, at 32 11008 x 4096 40.1 instead of 36.6).  Up to FEW_OWN_H tokens h is formed token by token beside
// the laying out, no launch of its own: 1024 x 2048, 8 adapters of 32 ranks, 256 tokens 26.8 us, by tiles of an adapter's tokens 36.2 (512 tokens 31.6 and
// 38.7, 1000 tokens 58.6 and 60.6: the margin shrinks with tokens x ranks).
constexpr int64_t FEW_DIRECT = 8, FEW_ALWAYS = 64, FEW_OWN_H = 256;

// Most tokens of a matrix: 64, or as many as make one round of workgroups (one a CU), two from 8 k-blocks on, three from 32 on.  A round takes
// some 10 us + 0.55 a k-block, tiles of 128 tokens 14 + 2.0 as long as they are no more than the CUs: 280 x 4864, 725 tokens (one round) 35 us, tiles 94;
// 384 x 1344, 1371 tokens (two, 14 k-blocks) 33 and 39; 3968 x 768, 300 tokens (three, 6) 38 and 28; 4096 x 4096, 300 tokens (three, 32) 66 and 83.
inline int64_t few_most(int64_t rows, int64_t cols, int32_t G) {
    const int64_t k_blocks = cols / (G % 128 == 0 ? 128 : G), rounds = k_blocks >= 32 ? 3 : (k_blocks >= 8 ? 2 : 1);
    const int64_t most = 256 * rounds / tokens_in(rows, PF_ROWS) * 64;
    return most > FEW_ALWAYS ? most : FEW_ALWAYS;
}
// Codes are read in whole pieces of 16 bytes, and units start on 16: a stream that ends between two (the last unit then may, too; the plan's layout
// leaves none such) is left to the kernels that read codes as they are.
inline bool few_fits(const PackArgs& P, int64_t T) {
    if (T > few_most(P.rows, P.cols, P.G) || (P.codes_bytes & 15) != 0) return false;
    return P.mask == nullptr && P.rows % 8 == 0 && (P.R_u == P.rows || P.R_u % PF_ROWS == 0) && (P.G % 128 == 0 || P.G == 96 || P.G == 64);
}

#ifdef __HIPCC__

// alpha_k B_k[row] . h_t
template <typename YT>
__device__ __forceinline__ float expand_one(const AdapterArgs& A, const float* __restrict__ h, int64_t t, int64_t row, int64_t rows) {
    const int32_t k = A.of[t];
    if (k < 0 || k >= A.n) return 0.0f;
    const int32_t rank = adapter_rank(A, k);
    const YT* __restrict__ const b = static_cast<const YT*>(A.b) + ((int64_t)k * rows + row) * A.max_rank;
    const float* __restrict__ const ht = h + t * A.max_rank;
    float sum = 0.0f;
#pragma unroll 2
    for (int32_t r = 0; r < rank; r += 8) {
        float bv[8], hv[8];
        load8(b + r, bv);
        load8(ht + r, hv);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (r + j < rank) sum = fmaf(bv[j], hv[j], sum);
    }
    return A.alpha != nullptr ? A.alpha[k] * sum : sum;
}

// Workgroups [0, shrinks): h, token by token; the others: X in the lanes' order, and its sums, one k-block and fragment a wavefront.
template <int S>
__global__ __launch_bounds__(256) void few_prepare_kernel(const FewArgs Q, const int64_t shrinks, float* __restrict__ h) {
    if (blockIdx.x < shrinks) {
        shrink_token(Q.X, Q.ldx, (int32_t)Q.P.cols, Q.A, false, h, blockIdx.x);
        return;
    }
    const int64_t at = (blockIdx.x - shrinks) * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, sub = lane & 31, hh = lane >> 5;
    const int32_t kb = (int32_t)(at / Q.fragments), n = (int32_t)(at - (int64_t)kb * Q.fragments);
    if (kb >= Q.n_kb) return;
    const int64_t t = n * 32 + sub;
    const bool in = t < Q.T;
    const uint16_t* const x = Q.X + (in ? t : 0) * Q.ldx + (int64_t)kb * (16 * S) + hh * (8 * S);
    float sum = 0.0f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const uint4 v = in ? *reinterpret_cast<const uint4*>(x + s * 8) : make_uint4(0u, 0u, 0u, 0u);
        Q.frag[(at * S + s) * 64 + lane] = v;
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = bf16_bits_to_f32(w[i] & 0xffffu) + __uint_as_float(w[i] & 0xffff0000u);
        sum += (p[0] + p[1]) + (p[2] + p[3]);
    }
    sum += __shfl_xor(sum, 32, 64);
    if (hh == 0) Q.xs[kb * Q.xs_ld + t] = sum;
}

template <int S, int NTF, int WAVES, bool LAID>
__global__ __launch_bounds__(WAVES * 64) void project_few_kernel(const FewArgs Q) {
    constexpr int CODES = 32 * 128 + 32;                   // bytes: 32 rows of a k-block's fields (or of a chunk's trits), and what a last octet reads past them
    constexpr int RED_BYTES = WAVES * NTF * 16 * 64 * 4;
    constexpr int BYTES = WAVES * CODES > RED_BYTES ? WAVES * CODES : RED_BYTES;
    __shared__ __attribute__((aligned(16))) char mem[BYTES];
    __shared__ float ab[WAVES][2][32];
    __shared__ uint16_t trits_of[256];
    for (int i = threadIdx.x; i < 256; i += WAVES * 64) trits_of[i] = (uint16_t)trit_fields(i);
    __syncthreads();
    const PackArgs& P = Q.P;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, sub = lane & 31, hh = lane >> 5;
    const uint32_t tb = blockIdx.x / Q.row_blocks;
    const int64_t row0 = (int64_t)(blockIdx.x - tb * Q.row_blocks) * PF_ROWS, t0 = (int64_t)tb * (NTF * 32);
    const int64_t rb = row0 / P.R_u, lrow0 = row0 - rb * P.R_u;
    const int32_t rows_left = P.R_u - lrow0 < PF_ROWS ? (int32_t)(P.R_u - lrow0) : PF_ROWS;
    const int32_t lr = sub < rows_left ? sub : rows_left - 1;
    const int32_t per_chunk = P.G / (16 * S);
    char* const mine = mem + wave * CODES;
    const uint32_t lds_codes = lds_address(mine);
    const uint32_t one = 0x3f803f80u;
    const bf16x8 ones = as_bf16x8(make_uint4(one, one, one, one));

    auto x_at = [&](int n, int32_t kb) {
        const int64_t t = t0 + n * 32 + sub;
        const int32_t f = (int32_t)tb * NTF + n;            // the last workgroup's second fragment may not exist
        return LAID ? Q.frag + (((int64_t)kb * Q.fragments + (f < Q.fragments ? f : Q.fragments - 1)) * S * 64 + lane)
                    : reinterpret_cast<const uint4*>(Q.X + (t < Q.T ? t : Q.T - 1) * Q.ldx + (int64_t)kb * (16 * S) + hh * (8 * S));
    };
    f32x16 tot[NTF] = {};
    float more = 0.0f;                                      // the adapters' part of a thread's first result
    // a k-block's treatment, known a k-block ahead
    int64_t base = 0;
    int a = 0;
    if (wave < Q.n_kb) a = __builtin_amdgcn_readfirstlane(pk_action(P, rb * P.n_chunks + wave / per_chunk, base));
    for (int32_t kb = wave; kb < Q.n_kb; kb += WAVES) {
        const int32_t j = kb / per_chunk, c = kb - j * per_chunk;
        const int64_t u = rb * P.n_chunks + j;
        const int64_t bpg = pk_bytes_per_group(a, P.G);
        const int kind = a;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // what was read of this place before
        int32_t stride = 0;                                 // bytes from row to row in LDS
        if (kind != 0) {
            const uint8_t* const from = P.codes + base + lrow0 * bpg;
            if (kind == 5 || per_chunk == 1) {              // whole rows, one behind the other
                stride = (int32_t)bpg;
                const int32_t most = (rows_left * stride + 15) / 16 - 1;       // up to 8 bytes past the unit: the stream has them
                for (int32_t i0 = 0; i0 * 16 < PF_ROWS * stride; i0 += 64)
                    lds_load16(lds_codes + i0 * 16, from + (i0 + lane < most ? i0 + lane : most) * 16);
            } else {                                        // 128 columns of wider rows: pieces of 16 bytes, as many as a code has bits
                const int b = (int)(bpg * 8 / P.G);
                stride = b * 16;
                for (int32_t i0 = 0; i0 < PF_ROWS * b; i0 += 64) {
                    const int32_t i = i0 + lane < rows_left * b ? i0 + lane : rows_left * b - 1;
                    lds_load16(lds_codes + i0 * 16, from + (i / b) * bpg + (c * b + i % b) * 16);
                }
            }
        }
        const int64_t g = u * P.R_u + lrow0 + lr;
        float alpha, beta, xsum[NTF];
        pk_affine(a, P.scale[g], P.offset[g], false, alpha, beta);
        uint4 x[S][NTF];
#pragma unroll
        for (int n = 0; n < NTF; ++n) {
            const uint4* const from = x_at(n, kb);
#pragma unroll
            for (int s = 0; s < S; ++s) x[s][n] = from[LAID ? s * 64 : s];
            if (LAID) xsum[n] = Q.xs[kb * Q.xs_ld + t0 + n * 32 + sub];
        }
        if (kb + WAVES < Q.n_kb) a = __builtin_amdgcn_readfirstlane(pk_action(P, rb * P.n_chunks + (kb + WAVES) / per_chunk, base));
        if (kb == wave && Q.h != nullptr) {                 // while all of this is on its way
            const int r = threadIdx.x & 31;
            const int64_t t = t0 + (threadIdx.x >> 5);
            if (r < rows_left && t < Q.T) more = expand_one<uint16_t>(Q.A, Q.h, t, row0 + r, P.rows);
        }
        if (hh == 0) {
            ab[wave][0][sub] = alpha;
            ab[wave][1][sub] = beta;
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        f32x16 acc[NTF] = {}, sums[LAID ? 1 : NTF] = {};
        const int64_t wcol = (int64_t)kb * (16 * S) + hh * (8 * S);
        auto steps = [&](auto octet) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const bf16x8 w = as_bf16x8(octet(s));
#pragma unroll
                for (int n = 0; n < NTF; ++n) {
                    acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, as_bf16x8(x[s][n]), acc[n], 0, 0, 0);
                    if (!LAID) sums[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ones, as_bf16x8(x[s][n]), sums[n], 0, 0, 0);
                }
            }
        };
        const char* const half = mine + lr * stride + hh * (stride >> 1);
        if (kind == 6) {
            steps([&](int s) { return fields1((uint32_t)(uint8_t)half[s]); });
        } else if (kind == 5) {
            const char* const trits = mine + lr * stride;
            steps([&](int s) {
                const uint32_t first = (uint32_t)(c * 2 * S + hh * S + s) * 8u, k = first / 5u, r = first - k * 5u;
                uint32_t v;
                __builtin_memcpy(&v, trits + k, 4);
                v = (uint32_t)trits_of[v & 0xffu] | (uint32_t)trits_of[(v >> 8) & 0xffu] << 10 | (uint32_t)trits_of[(v >> 16) & 0xffu] << 20;
                return fields2((v >> (2 * r)) & 0xffffu);
            });
        } else if (kind == 4) {
            steps([&](int s) { return fields2((uint32_t)*reinterpret_cast<const uint16_t*>(half + s * 2)); });
        } else if (kind == 3) {
            steps([&](int s) {
                uint32_t v;
                __builtin_memcpy(&v, half + s * 3, 4);
                return fields3(v & 0xffffffu);
            });
        } else if (kind == 2) {
            steps([&](int s) {
                uint32_t v;
                __builtin_memcpy(&v, half + s * 4, 4);
                return fields4(v);
            });
        } else if (kind == 1) {
            steps([&](int s) {
                uint2 v;
                __builtin_memcpy(&v, half + s * 8, 8);
                return fields8(v.x, v.y);
            });
        } else {
            steps([&](int s) { return skip_octet(P, rb * P.R_u + lrow0 + lr, wcol + s * 8, 0); });
            if (P.w_f32 != 0) {
#pragma unroll 1
                for (int term = 1; term < 3; ++term)
#pragma unroll 1
                    for (int s = 0; s < S; ++s) {           // rare: X once more from where it lies
                        const bf16x8 w = as_bf16x8(skip_octet(P, rb * P.R_u + lrow0 + lr, wcol + s * 8, term));
#pragma unroll
                        for (int n = 0; n < NTF; ++n) acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, as_bf16x8(x_at(n, kb)[LAID ? s * 64 : s]), acc[n], 0, 0, 0);
                    }
            }
        }
#pragma unroll
        for (int gr = 0; gr < 4; ++gr) {
            const float4 al = *reinterpret_cast<const float4*>(&ab[wave][0][gr * 8 + hh * 4]), be = *reinterpret_cast<const float4*>(&ab[wave][1][gr * 8 + hh * 4]);
            const float av[4] = {al.x, al.y, al.z, al.w}, bv[4] = {be.x, be.y, be.z, be.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int n = 0; n < NTF; ++n)
                    tot[n][gr * 4 + i] = fmaf(av[i], acc[n][gr * 4 + i], fmaf(bv[i], LAID ? xsum[n] : sums[LAID ? 0 : n][gr * 4 + i], tot[n][gr * 4 + i]));
        }
    }
    __syncthreads();
    float* const red = reinterpret_cast<float*>(mem);      // [WAVES][NTF * 16][64]
#pragma unroll
    for (int n = 0; n < NTF; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) red[((wave * NTF + n) * 16 + i) * 64 + lane] = tot[n][i];
    __syncthreads();
#pragma unroll 1
    for (int e = threadIdx.x; e < NTF * 1024; e += WAVES * 64) {
        const int r = e & 31, n = e >> 5;                  // neighbouring lanes: neighbouring rows of a token
        const int64_t y = row0 + r, t = t0 + n;
        if (r >= rows_left || t >= Q.T) continue;
        if (Q.h != nullptr && (e != (int)threadIdx.x || wave >= Q.n_kb)) more = expand_one<uint16_t>(Q.A, Q.h, t, y, P.rows);
        const int at = ((n >> 5) * 16 + (r >> 3) * 4 + (r & 3)) * 64 + ((r >> 2) & 1) * 32 + (n & 31);
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += red[w * NTF * 1024 + at];
        if (!isfinite(v)) v = (float)pk_slow_dot(P, y, Q.X + t * Q.ldx);
        Q.Y[t * Q.ldy + y] = (uint16_t)f32_to_bf16_bits(v + more);
    }
}

// h, or null: formed here (Q.h without it: there already).
template <int S>
int launch_few(FewArgs Q, float* h, hipStream_t st) {
    Q.fragments = (int32_t)tokens_in(Q.T, 32);
    Q.xs_ld = tokens_in(Q.T, 64) * 64;
    Q.row_blocks = (uint32_t)((Q.P.rows + PF_ROWS - 1) / PF_ROWS);
    const bool laid = Q.T > FEW_DIRECT;
    const int64_t wgs = (int64_t)Q.row_blocks * tokens_in(Q.T, Q.fragments == 1 ? 32 : 64);
    const int64_t shrinks = h != nullptr ? shrink_token_workgroups(Q.T, Q.A.max_rank) : 0;
    const int64_t ahead = shrinks + (laid ? tokens_in((int64_t)Q.n_kb * Q.fragments, 4) : 0);
    if (!fits_launch(wgs, 1024) || !fits_launch(ahead, 256)) return WINDQ_ESHAPE;
    if (ahead > 0) {
        few_prepare_kernel<S><<<dim3((uint32_t)ahead), dim3(256), 0, st>>>(Q, shrinks, h);
        if (hipGetLastError() != hipSuccess) return WINDQ_EHIP;
    }
    const dim3 g((uint32_t)wgs);
    if (!laid) project_few_kernel<S, 1, 16, false><<<g, dim3(1024), 0, st>>>(Q);
    else if (Q.fragments == 1) project_few_kernel<S, 1, 8, true><<<g, dim3(512), 0, st>>>(Q);
    else project_few_kernel<S, 2, 8, true><<<g, dim3(512), 0, st>>>(Q);
    return hipGetLastError() == hipSuccess ? WINDQ_OK : WINDQ_EHIP;
}

#endif  // __HIPCC__

}  // namespace windq
