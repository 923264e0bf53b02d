// Large products of a pair in half precision: 256 rows (of both) x 256 tokens a workgroup, eight wavefronts of 128 x 64 results, two a SIMD, so that one's matrix instructions go on
// while the other waits for its barrier or its operands: 11008 x 4096, 2048 tokens 417 -> 359 us (four wavefronts of 128 x 128, which read a third less
// from LDS, 417).  32 of the sum at a time, four buffers, three of them on their way; one barrier a buffer, ahead of its second step.  A row's four 16-byte
// slots are exchanged by bits 2 and 3 of the row.  LDS moves 128 bytes a clock where matrix instructions went without a pause, which is what it can;
// five buffers, priorities and the compiler's own order made no difference.
#pragma once

#include "windq_gemm.hpp"

namespace windq {

constexpr int GW_N = 256, GW_K = 32, GW_BUFFERS = 4, GW_THREADS = 512, GW_LOADS = (GM_MOST + GW_N) / 128;

// Tiles of 256 x 256 (pair_gemm_kernel) where their rounds of workgroups on 256 CUs take less time: 1.8 of the others' each, 3 of theirs where they are 128 wide.  A pair of
// 11008 x 4096, 2048 tokens (3 rounds and 6) 359 us and 417, 768 tokens (2 and 3) 273 and 265 with what comes ahead.
inline bool gemm_wide(int64_t large, int64_t tiles, int64_t by) { return 9 * ((large + 255) / 256) <= (by == 256 ? 5 : 3) * ((tiles + 255) / 256); }

#ifdef __HIPCC__

__global__ __launch_bounds__(GW_THREADS, 2) void pair_gemm_kernel(const GemmArgs Q) {
    constexpr int ROWS = GM_MOST + GW_N;                   // of a buffer, 64 bytes each
    __shared__ uint4 tile[GW_BUFFERS][ROWS * 4];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, sub = lane & 31, hh = lane >> 5;
    const int wm = wave & 1, wn = wave >> 1;
    // tiles of an XCD: a run, four columns of tiles wide
    const uint32_t n_tiles = gridDim.x, per = n_tiles >> 3;
    const uint32_t id = blockIdx.x < per * 8 ? (blockIdx.x & 7) * per + (blockIdx.x >> 3) : blockIdx.x;
    const uint32_t tall = (uint32_t)Q.tiles / Q.col_blocks, band = id / (4 * tall), inside = id - band * (4 * tall), width = Q.col_blocks - band * 4 < 4 ? Q.col_blocks - band * 4 : 4;
    const uint32_t tb = inside / width;
    const int64_t c0 = (int64_t)(band * 4 + inside - tb * width) * GM_MOST, t0 = (int64_t)tb * GW_N;
    const int32_t n_k = Q.K / GW_K;

    // A lane's share: slot (lane & 3) of rows 16 wave + lane / 4, 64 rows further on each time; slot p of row r holds the sixteen bytes of slot p ^ (r / 4 & 3).
    const int lr = wave * 16 + (lane >> 2), slot = (lane & 3) ^ ((lr >> 2) & 3);
    const uint16_t* const am = Q.wt + (c0 + lr) * Q.K + slot * 8;
    const uint16_t* bn[GW_N / 128];
#pragma unroll
    for (int i = 0; i < GW_N / 128; ++i) {
        const int64_t t = t0 + i * 128 + lr;
        bn[i] = Q.dY + (t < Q.T ? t : Q.T - 1) * Q.ldy + slot * 8;
    }
    const uint32_t lds = lds_address(tile);
    auto load = [&](int i, int32_t k, int buf) {
        const uint16_t* const from = i < GM_MOST / 128 ? am + (int64_t)i * 128 * Q.K : bn[i < GM_MOST / 128 ? 0 : i - GM_MOST / 128];
        lds_load16(lds + (buf * ROWS * 4 + i * 512 + wave * 64) * 16, from + k * GW_K);
    };
    const uint32_t arow = (wm * 128 + sub) * 64, brow = GM_MOST * 64 + (wn * 64 + sub) * 64;
    auto read_one = [&](int buf, int s, int i, f16x8 (&a)[4], f16x8 (&b)[2]) {
        const char* const at = reinterpret_cast<const char*>(tile[buf]) + (uint32_t)((2 * s + hh) ^ ((sub >> 2) & 3)) * 16;
        if (i < 2) b[i] = __builtin_bit_cast(f16x8, *reinterpret_cast<const uint4*>(at + brow + i * 32 * 64));
        else a[i - 2] = __builtin_bit_cast(f16x8, *reinterpret_cast<const uint4*>(at + arow + (i - 2) * 32 * 64));
    };
    f32x16 acc[4][2] = {};
#pragma unroll
    for (int p = 0; p < 3; ++p)
#pragma unroll
        for (int i = 0; i < GW_LOADS; ++i) load(i, p < n_k ? p : n_k - 1, p);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * GW_LOADS) : "memory");
    __syncthreads();
    f16x8 a[2][4], b[2][2];
#pragma unroll
    for (int i = 0; i < 6; ++i) read_one(0, 0, i, a[0], b[0]);
    for (int32_t k = 0; k < n_k; ++k) {
        const int buf = k & 3, next = (k + 1) & 3, then = (k + 3) & 3;
        const int32_t k3 = k + 3 < n_k ? k + 3 : n_k - 1;  // past the end: again the last, into a buffer that nobody reads
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                acc[i >> 1][i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[s][i >> 1], b[s][i & 1], acc[i >> 1][i & 1], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
                if (s == 1 && i == 0) {
                    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * GW_LOADS) : "memory");     // the next buffer's loads are done, this one's reads too
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                }
                if (i < 6) read_one(s == 0 ? buf : next, s == 0 ? 1 : 0, i, a[s ^ 1], b[s ^ 1]);
                if (s == 0 && i < GW_LOADS) load(i, k3, then);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    pair_tile<4, GW_THREADS>(Q, acc, reinterpret_cast<uint16_t*>(tile), c0, t0, wm, wn, tid);
}

#endif  // __HIPCC__

}  // namespace windq
