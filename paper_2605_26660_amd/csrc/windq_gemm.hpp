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

#include "windq_adapters.hpp"

namespace windq {

constexpr int GM_MOST = 256, GM_N = 128, GM_K = 64, GM_THREADS = 256, GM_BUFFERS = 3;

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

template <int MF>                                          // fragments of a wavefront along the columns
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
