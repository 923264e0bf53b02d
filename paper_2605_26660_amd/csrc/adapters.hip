// Tokens grouped by adapter, and h = A x (or dh = alpha B^T dY) for many tokens of bfloat16.
#include "windq_adapters.hpp"

namespace windq {

__global__ __launch_bounds__(256) void group_kernel(const GroupArgs Q) { group_adapter(Q, blockIdx.x); }

int launch_group(const GroupArgs& G, hipStream_t st) {
    if (!fits_launch(G.n, 256)) return WINDQ_ESHAPE;
    group_kernel<<<dim3((uint32_t)G.n), dim3(256), 0, st>>>(G);
    return hipGetLastError() == hipSuccess ? WINDQ_OK : WINDQ_EHIP;
}

// 64 tokens of one adapter by up to 16 RF ranks, over a piece of the columns that the four wavefronts share 64 at a time.  Both factors
// are rows along the sum's axis, so operands come straight from memory; ranks are the M side.  Bound by reading X once:
// 2048 tokens of 4096 and of 11008 columns by 64 ranks, both in one launch, 28 to 32 us (82 MB read past L2).
template <int RF>
__global__ __launch_bounds__(256) void shrink_kernel(const ShrinkArgs Q1, const ShrinkArgs Q2, const int64_t first2, const int64_t first) {
    __shared__ float red[4][RF * 16][65];
    const int64_t id = first + blockIdx.x;
    const ShrinkArgs& Q = id < first2 ? Q1 : Q2;
    const int64_t block = id < first2 ? id : id - first2;
    const int64_t slot = block / Q.splits;
    const int32_t split = (int32_t)(block - slot * Q.splits);
    const int32_t k = Q.owner[slot];
    if (k < 0) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, sub = lane & 15, q = lane >> 4;
    const int32_t rank = adapter_rank(Q.A, k);
    const int32_t steps = (Q.width + 63) / 64, per = (steps + Q.splits - 1) / Q.splits;
    const int32_t s0 = split * per, s1 = s0 + per < steps ? s0 + per : steps;
    const uint16_t* xp[4];
    const int32_t some = Q.place[slot * GROUP];            // a slot in use holds a token at its start
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const int32_t t = Q.place[slot * GROUP + n * 16 + sub];
        xp[n] = static_cast<const uint16_t*>(Q.X) + (int64_t)(t < 0 ? some : t) * Q.ld + q * 8;
    }
    const uint16_t* ap[RF];
#pragma unroll
    for (int f = 0; f < RF; ++f) {
        const int32_t r = f * 16 + sub;
        ap[f] = static_cast<const uint16_t*>(Q.a) + ((int64_t)k * Q.A.max_rank + (r < rank ? r : 0)) * Q.lda + q * 8;
    }
    f32x4 acc[RF][4] = {};
    if (rank > 0) {
        // 64 columns, a row's cache line, in two instructions each
        const uint4 none = make_uint4(0u, 0u, 0u, 0u);
        for (int32_t s = s0 + wave; s < s1; s += 4) {
            uint4 a[2][RF], b[2][4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bool in = s * 64 + u * 32 + q * 8 < Q.width;
                const int64_t c = in ? s * 64 + u * 32 : -q * 8;          // past the end the row's start, counted as zeros
#pragma unroll
                for (int n = 0; n < 4; ++n) b[u][n] = *reinterpret_cast<const uint4*>(xp[n] + c);
#pragma unroll
                for (int f = 0; f < RF; ++f) {
                    a[u][f] = *reinterpret_cast<const uint4*>(ap[f] + c);
                    if (!in) a[u][f] = none;
                }
#pragma unroll
                for (int n = 0; n < 4; ++n)
                    if (!in) b[u][n] = none;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int f = 0; f < RF; ++f)
#pragma unroll
                    for (int n = 0; n < 4; ++n)
                        acc[f][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a[u][f]), as_bf16x8(b[u][n]), acc[f][n], 0, 0, 0);
        }
    }
#pragma unroll
    for (int f = 0; f < RF; ++f)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) red[wave][f * 16 + q * 4 + i][n * 16 + sub] = acc[f][n][i];
    __syncthreads();
    float* __restrict__ const out = Q.part + ((int64_t)split * Q.slots + slot) * GROUP * (RF * 16);
    for (int e = threadIdx.x; e < GROUP * RF * 16; e += 256) {
        const int r = e / GROUP, n = e % GROUP;
        out[e] = r < rank ? ((red[0][r][n] + red[1][r][n]) + red[2][r][n]) + red[3][r][n] : 0.0f;
    }
}

int launch_shrink(const ShrinkArgs& S, const ShrinkArgs* more, hipStream_t st) {
    const ShrinkArgs& S2 = more != nullptr ? *more : S;
    const int64_t first2 = S.slots * S.splits, wgs = first2 + (more != nullptr ? S2.slots * S2.splits : 0);
    const dim3 b(256);
    return launch_pieces(wgs, 256, [&](int64_t first, dim3 g) {
        switch (shrink_ranks(S.A.max_rank) / 16) {
            case 1: shrink_kernel<1><<<g, b, 0, st>>>(S, S2, first2, first); break;
            case 2: shrink_kernel<2><<<g, b, 0, st>>>(S, S2, first2, first); break;
            case 3: shrink_kernel<3><<<g, b, 0, st>>>(S, S2, first2, first); break;
            case 4: shrink_kernel<4><<<g, b, 0, st>>>(S, S2, first2, first); break;
            case 5: shrink_kernel<5><<<g, b, 0, st>>>(S, S2, first2, first); break;
            case 6: shrink_kernel<6><<<g, b, 0, st>>>(S, S2, first2, first); break;
            case 7: shrink_kernel<7><<<g, b, 0, st>>>(S, S2, first2, first); break;
            default: shrink_kernel<8><<<g, b, 0, st>>>(S, S2, first2, first); break;
        }
    });
}

// A workgroup adds up eight ranks of a slot's pieces; the workgroups behind them write the zeros of tokens without an adapter, 64 tokens each.
constexpr int JOIN_RANKS = 8;
__global__ __launch_bounds__(256) void join_kernel(const JoinArgs Q1, const JoinArgs Q2, const int64_t first2, const int64_t first) {
    const int64_t id = first + blockIdx.x;
    const JoinArgs& Q = id < first2 ? Q1 : Q2;
    const int64_t block = id < first2 ? id : id - first2;
    const int32_t R = Q.A.max_rank, ranks = (R + 15) / 16 * 16, groups = R / JOIN_RANKS;
    const int64_t slot = block / groups;
    if (slot >= Q.slots) {
        const int64_t t0 = (block - Q.slots * groups) * GROUP;
        for (int e = threadIdx.x; e < GROUP * R; e += 256) {
            const int64_t t = t0 + e / R;
            if (t >= Q.T) break;
            const int32_t id = Q.A.of[t];
            if (id < 0 || id >= Q.A.n) Q.h[t * R + e % R] = 0.0f;
        }
        return;
    }
    __shared__ float tile[GROUP][JOIN_RANKS + 1];          // places by ranks, for h
    const int32_t k = Q.owner[slot];
    if (k < 0) return;
    const int64_t places = Q.slots * GROUP;
    const int32_t r0 = (int32_t)(block - slot * groups) * JOIN_RANKS;
    const int n = threadIdx.x & 63;                        // places side by side
    const int32_t t = Q.place[slot * GROUP + n];
    const float factor = Q.scaled && Q.A.alpha != nullptr ? Q.A.alpha[k] : 1.0f;
#pragma unroll
    for (int i = 0; i < JOIN_RANKS / 4; ++i) {
        const int r = r0 + i * 4 + (threadIdx.x >> 6);
        const float* __restrict__ const p = Q.part + (slot * ranks + r) * GROUP + n;
        float v = 0.0f;
        if (Q.given != nullptr) {
            if (t >= 0) v = Q.given[(int64_t)t * R + r];
        } else {
#pragma unroll 8
            for (int32_t s = 0; s < Q.splits; ++s) v += p[(int64_t)s * places * ranks];
        }
        v = t >= 0 ? factor * v : 0.0f;
        tile[n][r - r0] = v;
        if (Q.planes != nullptr) {
            uint32_t hi, mid, lo;
            split3(v, hi, mid, lo);
            uint16_t* __restrict__ const o = Q.planes + r * places + slot * GROUP + n;
            o[0] = (uint16_t)hi;
            o[R * places] = (uint16_t)mid;
            o[2 * R * places] = (uint16_t)lo;
        }
    }
    if (Q.h == nullptr) return;
    __syncthreads();
    for (int e = threadIdx.x; e < GROUP * JOIN_RANKS; e += 256) {
        const int32_t to = Q.place[slot * GROUP + e / JOIN_RANKS];
        if (to >= 0) Q.h[(int64_t)to * R + r0 + e % JOIN_RANKS] = tile[e / JOIN_RANKS][e % JOIN_RANKS];
    }
}

int launch_join(const JoinArgs& J, const JoinArgs* more, hipStream_t st) {
    auto count = [](const JoinArgs& j) { return j.slots * (j.A.max_rank / JOIN_RANKS) + (j.h != nullptr ? tokens_in(j.T, GROUP) : 0); };
    const int64_t first2 = count(J), wgs = first2 + (more != nullptr ? count(*more) : 0);
    return launch_pieces(wgs, 256, [&](int64_t first, dim3 g) { join_kernel<<<g, dim3(256), 0, st>>>(J, more != nullptr ? *more : J, first2, first); });
}

}  // namespace windq
