// Low-rank adapters beside a packed product: kernels that the way there and the way back share.
#pragma once

#include "windq_project.hpp"

namespace windq {

inline int64_t tokens_in(int64_t T, int64_t by) { return (T + by - 1) / by; }

// Kernels count a side's values in 32 bits, some of them up to a step past its end; and no tensor of more than 2^40 values fits a card, so that
// bytes counted from what is left never pass 64 bits.
constexpr int64_t MOST_SIDE = ((int64_t)1 << 31) - 512, MOST_VALUES = (int64_t)1 << 40;
inline bool sizes_fit(int64_t T, int64_t rows, int64_t cols, int32_t n, int32_t max_rank) {
    if (T > ((int64_t)1 << 31) - 1 || rows > MOST_SIDE || cols > MOST_SIDE || n > WINDQ_MAX_ADAPTERS || max_rank > WINDQ_MAX_RANK) return false;
    const int64_t wide = rows > cols ? rows : cols;
    return rows * cols <= MOST_VALUES && T * wide <= MOST_VALUES && (int64_t)n * max_rank * wide <= MOST_VALUES;
}
inline bool grad_sizes_fit(int64_t T, int64_t rows, int64_t cols) { return T * rows <= (int64_t)0x7fffffff && T * cols <= (int64_t)0x7fffffff; }

// A launch of any number of workgroups, in pieces where one would hold 2^32 threads: launch(first, count).
template <typename Launch>
inline int launch_pieces(int64_t workgroups, int64_t threads, Launch launch) {
    const int64_t most = (int64_t)0xffffffff / threads;
    for (int64_t first = 0; first < workgroups; first += most) {
        launch(first, dim3((uint32_t)(workgroups - first < most ? workgroups - first : most)));
        if (hipGetLastError() != hipSuccess) return WINDQ_EHIP;
    }
    return WINDQ_OK;
}

// The tokens of adapter k in their own order, at places that start with a multiple of GROUP: place[] holds tokens, -1 where there is none.
// Adapter k's first slot of GROUP places is (tokens of adapters below it) / GROUP + k: slots never overlap, and no adapter
// has to wait for the counts of the others.
constexpr int GROUP = 64;
inline int64_t group_slots(int64_t T, int32_t n) { return T / GROUP + n + 1; }

struct GroupArgs {
    const int32_t* of;
    int64_t T;
    int32_t n;
    int64_t slots;
    int32_t* place;            // [slots * GROUP]
    int32_t* owner;            // [slots] adapter, or -1: an empty slot
    int32_t* first;            // [n] first place of an adapter
    int32_t* count;            // [n] its tokens
};

// Up to so many tokens h is formed token by token, one launch instead of three: 1024 x 1600 in chunks of 160, 8 adapters of 32 ranks, 64 tokens 16.3 us in
// all and 27.1 (128 tokens 23.0 and 32.7, 512 tokens 66.5 and 71.8: the margin shrinks with tokens x ranks).
constexpr int64_t SHRINK_FEW = 64;

// Sums of x_t a_r over pieces of the columns, tile by tile of one adapter's tokens.
struct ShrinkArgs {
    const void* X;             // [T][ld]
    int64_t ld;
    const void* a;             // [n][max_rank][lda]
    int64_t lda;
    int32_t width;             // columns, a multiple of 8
    int32_t splits;
    int64_t slots;
    const int32_t* place;
    const int32_t* owner;
    AdapterArgs A;
    float* part;               // [splits][slots][ranks][GROUP], ranks = max_rank rounded up to 16
};

// The pieces added up: h (times alpha where scaled) by token, and by place as three bfloat16 terms, transposed.
struct JoinArgs {
    const float* part;
    int32_t splits;
    int64_t slots;
    const int32_t* place;
    const int32_t* owner;
    int64_t T;
    AdapterArgs A;
    bool scaled;
    float* h;                  // [T][max_rank], or null
    uint16_t* planes;          // [3][max_rank][slots * GROUP], or null
    const float* given;        // [T][max_rank] h in the pieces' place, or null
};

int launch_group(const GroupArgs& G, hipStream_t st);
int launch_shrink(const ShrinkArgs& S, const ShrinkArgs* more /* or null */, hipStream_t st);    // bfloat16; both of one max_rank
int launch_join(const JoinArgs& J, const JoinArgs* more /* or null */, hipStream_t st);
inline int32_t shrink_ranks(int32_t max_rank) { return (max_rank + 15) / 16 * 16; }
// Enough pieces that the launch has some workgroups for every CU, and a wavefront at least 64 columns: the way back of 2048 tokens of one adapter through
// 11008 x 4096 takes 267 us in all and 316 without pieces, 700 tokens of 16 adapters through 4096 x 4096 82 and 92 (256 in the place of 512: the same).
inline int32_t shrink_splits(int64_t slots, int64_t width) {
    int64_t s = 512 / slots;
    if (s > width / 256) s = width / 256;
    return (int32_t)(s < 1 ? 1 : (s > 32 ? 32 : s));
}
// Most slots x splits of as many slots or fewer: a workspace sized for more tokens does for fewer.
inline int64_t shrink_pieces(int64_t slots, int64_t width) {
    const int64_t splits = width / 256 < 32 ? width / 256 : 32;
    const int64_t most = slots * splits < 512 ? slots * splits : 512;
    return most > slots ? most : slots;
}
// Floats of ShrinkArgs::part for sums over so many columns: the width that is launched, B transposed and dY have their rows in eights.
inline size_t shrink_floats(int64_t slots, int64_t width, int32_t max_rank) { return (size_t)shrink_pieces(slots, width) * GROUP * (size_t)shrink_ranks(max_rank); }
inline int64_t in_eights(int64_t rows) { return (rows + 7) / 8 * 8; }

#ifdef __HIPCC__

// A workgroup per adapter: counts its tokens and those of the adapters below it, then lists its own, in ascending order.
__device__ __forceinline__ void group_adapter(const GroupArgs& Q, const int32_t k) {
    __shared__ int32_t sums[2][4];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int32_t below = 0, mine = 0;
    for (int64_t t = threadIdx.x; t < Q.T; t += 256) {
        const int32_t id = Q.of[t];
        below += id >= 0 && id < k ? 1 : 0;
        mine += id == k ? 1 : 0;
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
        below += __shfl_xor(below, m, 64);
        mine += __shfl_xor(mine, m, 64);
    }
    if (lane == 0) {
        sums[0][wave] = below;
        sums[1][wave] = mine;
    }
    __syncthreads();
    below = sums[0][0] + sums[0][1] + sums[0][2] + sums[0][3];
    mine = sums[1][0] + sums[1][1] + sums[1][2] + sums[1][3];
    const int64_t slot = (int64_t)(below / GROUP) + k;
    const int64_t end = k + 1 == Q.n ? Q.slots : (int64_t)((below + mine) / GROUP) + k + 1;
    if (threadIdx.x == 0) {
        Q.first[k] = (int32_t)(slot * GROUP);
        Q.count[k] = mine;
    }
    const int64_t used = slot + (mine + GROUP - 1) / GROUP;
    for (int64_t s = slot + threadIdx.x; s < end; s += 256) Q.owner[s] = s < used ? k : -1;
    int64_t at = slot * GROUP;
    __syncthreads();
    for (int64_t t0 = 0; t0 < Q.T; t0 += 256) {
        const int64_t t = t0 + threadIdx.x;
        const bool hit = t < Q.T && Q.of[t] == k;
        const uint64_t hits = __ballot(hit);
        if (lane == 0) sums[0][wave] = __popcll(hits);
        __syncthreads();
        int32_t before = __popcll(hits & ((1ull << lane) - 1ull)), all = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            before += w < wave ? sums[0][w] : 0;
            all += sums[0][w];
        }
        if (hit) Q.place[at + before] = (int32_t)t;
        at += all;
        __syncthreads();
    }
    for (int64_t p = at + threadIdx.x; p < end * GROUP; p += 256) Q.place[p] = -1;
}

// ------------------------------------------------------------------------------------------------ h = A x, token by token
// (On the way back: dh = alpha B^T dY, with B transposed in A's place.)  A wavefront per token and rank, eight columns a lane at a time: bound by latency,
// so as many wavefronts as there are, and eight loads on their way.
template <typename XT>
__device__ __forceinline__ void load8(const XT* __restrict__ p, float (&v)[8]) {
    if constexpr (sizeof(XT) == 4) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
        const uint4 r = *reinterpret_cast<const uint4*>(p);
        v[0] = bf16_bits_to_f32(r.x & 0xffffu); v[1] = __uint_as_float(r.x & 0xffff0000u);
        v[2] = bf16_bits_to_f32(r.y & 0xffffu); v[3] = __uint_as_float(r.y & 0xffff0000u);
        v[4] = bf16_bits_to_f32(r.z & 0xffffu); v[5] = __uint_as_float(r.z & 0xffff0000u);
        v[6] = bf16_bits_to_f32(r.w & 0xffffu); v[7] = __uint_as_float(r.w & 0xffff0000u);
    }
}

constexpr int SHRINK_RANKS = 4;                           // of a workgroup
template <typename XT>
__device__ __forceinline__ void shrink_token(const XT* __restrict__ X, int64_t ldx, int32_t cols, const AdapterArgs& A, bool scaled, float* __restrict__ h, uint32_t block) {
    const uint32_t groups = (uint32_t)A.max_rank / SHRINK_RANKS;
    const int64_t t = block / groups;
    const int32_t r = (int32_t)(block - (uint32_t)t * groups) * SHRINK_RANKS + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int32_t k = A.of[t];
    const int32_t rank = k < 0 || k >= A.n ? 0 : adapter_rank(A, k);
    float sum = 0.0f;
    if (r < rank) {
        const XT* __restrict__ const a = static_cast<const XT*>(A.a) + ((int64_t)k * A.max_rank + r) * cols;
        const XT* __restrict__ const x = X + t * ldx;
        float acc[2] = {0.0f, 0.0f};
#pragma unroll 4
        for (int32_t c = lane * 8; c < cols; c += 512) {
            float xv[8], av[8];
            load8(x + c, xv);
            load8(a + c, av);
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j & 1] = fmaf(av[j], xv[j], acc[j & 1]);
        }
        sum = acc[0] + acc[1];
        if (scaled && A.alpha != nullptr) sum *= A.alpha[k];
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) sum += __shfl_xor(sum, m, 64);
    if (lane == 0) h[t * A.max_rank + r] = sum;
}

inline int64_t shrink_token_workgroups(int64_t T, int32_t max_rank) { return T * (max_rank / SHRINK_RANKS); }

template <typename XT>
__global__ __launch_bounds__(256) void shrink_token_kernel(const XT* __restrict__ X, int64_t ldx, int32_t cols, const AdapterArgs A, bool scaled, float* __restrict__ h) {
    shrink_token(X, ldx, cols, A, scaled, h, blockIdx.x);
}

template <typename XT>
int launch_shrink_token(const XT* X, int64_t ldx, int64_t T, int32_t cols, const AdapterArgs& A, bool scaled, float* h, hipStream_t st) {
    const int64_t most = (int64_t)0xffffff / (A.max_rank / SHRINK_RANKS);      // tokens of a launch: less than 2^32 threads
    for (int64_t t = 0; t < T; t += most) {
        AdapterArgs here = A;
        here.of = A.of + t;
        const int64_t wgs = shrink_token_workgroups(T - t < most ? T - t : most, A.max_rank);
        shrink_token_kernel<XT><<<dim3((uint32_t)wgs), dim3(256), 0, st>>>(X + t * ldx, ldx, cols, here, scaled, h + t * A.max_rank);
        if (hipGetLastError() != hipSuccess) return WINDQ_EHIP;
    }
    return WINDQ_OK;
}

__device__ __forceinline__ uint4 pack8(const uint32_t (&w)[8]) {
    return make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
}

// What the adapters of a wavefront's 64 tokens add to a tile of 32 M rows x 64 tokens of 32x32x16 results (alpha_k B_k h_t, or A_k^T dh_t): for each
// adapter among the tokens, its factors against its own tokens' h and the others' zeros.  row_of(f): where a lane's factors of
// fragment f begin, k given; h [T][max_rank] times `scaled`'s alpha.  In bfloat16 h enters as two bfloat16 terms: 16 of its 24 bits, 2^8 finer
// than the results' rounding, for two instructions instead of three (fp32: three terms, and of the factors too).
template <typename YT, int M, typename Rows>
__device__ __forceinline__ void add_adapters(const AdapterArgs& A, const float* __restrict__ h, bool scaled, int64_t t0, int64_t T, int lane, Rows row_of,
                                             f32x16 (&tot)[M][2]) {
    constexpr int TA = sizeof(YT) == 4 ? 3 : 1, TH = sizeof(YT) == 4 ? 3 : 2;
    const int sub = lane & 31, hh = lane >> 5;
    const int32_t id = t0 + lane < T ? A.of[t0 + lane] : -1;
    uint64_t left = __ballot(id >= 0 && id < A.n);
    while (left != 0) {
        const int32_t k = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        const uint64_t mine = __ballot(id == k);
        left &= ~mine;
        const int32_t rank = adapter_rank(A, k);
        const float factor = scaled && A.alpha != nullptr ? A.alpha[k] : 1.0f;
        for (int32_t r0 = 0; r0 < rank; r0 += 16) {
            const int32_t r = r0 + hh * 8;
            uint4 bt[TH][2], at[TA][M];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const bool has = ((mine >> (n * 32 + sub)) & 1ull) != 0 && r < rank;
                float v[8] = {};
                if (has) load8(h + (t0 + n * 32 + sub) * A.max_rank + r, v);
                uint32_t w[3][8];
#pragma unroll
                for (int i = 0; i < 8; ++i) split3(has && r + i < rank ? factor * v[i] : 0.0f, w[0][i], w[1][i], w[2][i]);      // a factor that is not finite: its own tokens' alone
#pragma unroll
                for (int m = 0; m < TH; ++m) bt[m][n] = pack8(w[m]);
            }
            bool broken = false;
#pragma unroll
            for (int f = 0; f < M; ++f) {
                float v[8] = {};
                if (r < rank) load8(row_of(k, f) + r, v);
                uint32_t w[3][8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float x = r + i < rank ? v[i] : 0.0f;
                    broken |= !isfinite(x);
                    if (TA == 1) w[0][i] = __float_as_uint(x) >> 16;
                    else split3(x, w[0][i], w[1][i], w[2][i]);
                }
#pragma unroll
                for (int m = 0; m < TA; ++m) at[m][f] = pack8(w[m]);
            }
            if (__any(broken)) {                            // times the other tokens' zeros they would be NaN: kept apart
#pragma unroll
                for (int f = 0; f < M; ++f)
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        f32x16 own = {};
#pragma unroll
                        for (int ma = 0; ma < TA; ++ma)
#pragma unroll
                            for (int mh = 0; mh < TH; ++mh)
                                if (ma + mh < 3) own = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(at[ma][f]), as_bf16x8(bt[mh][n]), own, 0, 0, 0);
                        const bool in = ((mine >> (n * 32 + sub)) & 1ull) != 0;
#pragma unroll
                        for (int i = 0; i < 16; ++i) tot[f][n][i] += in ? own[i] : 0.0f;
                    }
                continue;
            }
#pragma unroll
            for (int ma = 0; ma < TA; ++ma)
#pragma unroll
                for (int mh = 0; mh < TH; ++mh)
                    if (ma + mh < 3) {
#pragma unroll
                        for (int f = 0; f < M; ++f)
#pragma unroll
                            for (int n = 0; n < 2; ++n)
                                tot[f][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(at[ma][f]), as_bf16x8(bt[mh][n]), tot[f][n], 0, 0, 0);
                    }
        }
    }
}

// Direct loads to LDS: lane l's 16 (or 4) bytes go to `to` + 16 l (4 l); `to` is the same for the wavefront.  Written out because the compiler
// would have every later read of LDS wait for them, whatever it reads; here whoever reads waits for vmcnt and a barrier first.
__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return (uint32_t)reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) void*)p);
}
__device__ __forceinline__ void lds_load16(uint32_t to, const void* from) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(from) : "memory");
}
__device__ __forceinline__ void lds_load4(uint32_t to, const void* from) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(from) : "memory");
}

#endif  // __HIPCC__

}  // namespace windq
