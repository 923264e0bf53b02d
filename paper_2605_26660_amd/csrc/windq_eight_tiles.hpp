// Products of many 8-bit tokens with a plan laid out for them: tiles of 64 WR rows x 64 WT tokens (of a pair: 32 WR rows of both).
#pragma once

#include "windq_eight.hpp"

namespace windq {

#ifdef __HIPCC__

// A lane's fields of one row block and k-block.
template <int S>
struct EightRaw {
    uint32_t v[4 * S];
    __device__ __forceinline__ void load(int kind, const char* __restrict__ fields, int lane) {
        if (kind == 6) {
            __builtin_memcpy(v, fields + lane * (4 * ((S + 1) / 2)), 4 * ((S + 1) / 2));
        } else if (kind == 4) {
            __builtin_memcpy(v, fields + lane * (4 * S), 4 * S);
        } else if (kind == 2) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const uint2 w = reinterpret_cast<const uint2*>(fields)[s * 64 + lane];
                v[2 * s] = w.x;
                v[2 * s + 1] = w.y;
            }
        } else if (kind == 1) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const uint4 w = reinterpret_cast<const uint4*>(fields)[s * 64 + lane];
                v[4 * s] = w.x;
                v[4 * s + 1] = w.y;
                v[4 * s + 2] = w.z;
                v[4 * s + 3] = w.w;
            }
        }
    }
    template <int KIND>
    __device__ __forceinline__ void operands(i32x4 (&w)[S]) const {
#pragma unroll
        for (int s = 0; s < S; ++s) w[s] = operand<KIND>(s);
    }
    template <int KIND>
    __device__ __forceinline__ i32x4 operand(int s) const {
        if constexpr (KIND == 6) return eight_fields1(v[s >> 1], s & 1);
        else if constexpr (KIND == 4) return eight_fields2(v[s]);
        else if constexpr (KIND == 2) return eight_fields4(make_uint2(v[2 * s], v[2 * s + 1]));
        else return as_i32x4(make_uint4(v[4 * s], v[4 * s + 1], v[4 * s + 2], v[4 * s + 3]));
    }
};

template <int V>
struct Const {
    static constexpr int value = V;
};

template <typename YT, int S, int WR, int WT, bool PAIR>
__global__ __launch_bounds__(WR* WT * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void eight_tiles_kernel(const EightArgs Q, const uint32_t row_tiles) {
    constexpr int TOKENS = WT * 64, LOADS = 8 / WR;
    __shared__ uint4 xt[2][TOKENS * 8];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, sub = lane & 31, hh = lane >> 5;
    const int wr = wave % WR, wt = wave / WR;
    const bool w_f32 = Q.w_f32 != 0;
    // Consecutive workgroups land on the eight XCDs in turn; each XCD gets a run of tiles that share tokens.
    const uint32_t n_tiles = gridDim.x, per = n_tiles >> 3;
    const uint32_t tile = blockIdx.x < per * 8 ? (blockIdx.x & 7) * per + (blockIdx.x >> 3) : blockIdx.x;
    const uint32_t tb = tile / row_tiles;
    const int64_t b0 = (int64_t)(tile - tb * row_tiles) * WR + wr, t0 = (int64_t)tb * TOKENS;
    const int32_t n_kb = Q.n_kb;

    // a wavefront's two row blocks: neighbours, or the same of the gate and of the up; past the last one: computed for nothing, stored by nobody
    int64_t b[2], rb[2], in[2];
    const char* image[2];
    const float* affine[2];
#pragma unroll
    for (int f = 0; f < 2; ++f) {
        b[f] = PAIR ? b0 : 2 * b0 + f;
        const int64_t at = b[f] < Q.NB ? b[f] : Q.NB - 1;
        rb[f] = at / Q.RB;
        in[f] = at - rb[f] * Q.RB;
        image[f] = Q.P[PAIR ? f : 0].image;
        affine[f] = reinterpret_cast<const float*>(image[f] + Q.affine) + at * Q.n_chunks * 64 + sub;
    }

    // X: a row of 128 bytes a token, eight slots; slot p of token n holds slot p ^ (n / 2 & 7)
    const int8_t* xsrc[LOADS];
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
        const int n = (k * WR * WT + wave) * 8 + (lane >> 3), slot = (lane & 7) ^ ((n >> 1) & 7);
        const int64_t t = t0 + n < Q.T ? t0 + n : Q.T - 1;
        xsrc[k] = Q.codes + t * Q.width + (slot < 2 * S ? slot : 0) * 16;
    }
    const uint32_t lds_xt = lds_address(xt);
    auto load_x = [&](int32_t kb, int buf) {
#pragma unroll
        for (int k = 0; k < LOADS; ++k) lds_load16(lds_xt + (buf * (TOKENS * 8) + (k * WR * WT + wave) * 64) * 16, xsrc[k] + (int64_t)kb * (32 * S));
    };
    const int32_t* sums[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const int64_t t = t0 + wt * 64 + n * 32 + sub;
        sums[n] = Q.sums + (t < Q.T ? t : Q.T - 1) * Q.sums_ld;
    }

    struct Unit {
        const char* fields;
        int kind;
    };
    auto unit_of = [&](int f, int32_t kb) {
        const int32_t j = kb / Q.per_chunk, c = kb - j * Q.per_chunk;
        const EightUnit u = eight_unit(Q.P[PAIR ? f : 0], rb[f] * Q.n_chunks + j, Q.RB * Q.per_chunk, S, w_f32);
        const int kind = __builtin_amdgcn_readfirstlane(u.kind);
        return Unit{u.fields + (in[f] * Q.per_chunk + c) * eight_bytes(kind, S, w_f32), kind};
    };

    f32x16 tot[2][2] = {};
    i32x16 acc[2][2] = {};
    EightRaw<S> raw[2];
    Unit now[2];
    float alpha[2], behind = 0.0f;                         // of the k-block; of the second row block's sums that are still to be added up
#pragma unroll
    for (int f = 0; f < 2; ++f) {
        now[f] = unit_of(f, 0);
        raw[f].load(now[f].kind, now[f].fields, lane);
        alpha[f] = now[f].kind == 0 || now[f].kind == 7 ? 0.0f : affine[f][0];
    }
    load_x(0, 0);
    float pair_beta[2] = {}, pair_sum[2] = {};

    for (int32_t kb = 0; kb < n_kb; ++kb) {
        const int buf = kb & 1;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const int32_t then = kb + 1 < n_kb ? kb + 1 : kb;
        load_x(then, buf ^ 1);
        // beta times the tokens' sums, two k-blocks an instruction: a lane's half has one of them
        const bool both = (kb & 1) != 0 || kb + 1 == n_kb;
        if (both) {
            const int32_t at = (kb & ~1) + hh;
            const bool valid = at < n_kb;
            const int32_t j = (valid ? at : kb) / Q.per_chunk;
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                const float v = affine[f][j * 64 + 32];
                pair_beta[f] = valid ? v : 0.0f;
            }
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const int32_t v = sums[n][valid ? at : kb];
                pair_sum[n] = valid ? (float)v : 0.0f;
            }
        }
        uint4 x[S][2];
        const char* const xb = reinterpret_cast<const char*>(xt[buf]) + (wt * 64 + sub) * 128;
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int n = 0; n < 2; ++n) x[s][n] = *reinterpret_cast<const uint4*>(xb + n * 32 * 128 + (((2 * s + hh) ^ ((sub >> 1) & 7)) << 4));

        auto phase = [&](auto F) {
            constexpr int f = decltype(F)::value, other = f ^ 1;
            const float fold = f == 0 ? behind : alpha[0];
            auto add_up = [&](int from, int count) {        // of the other row block's results
#pragma unroll
                for (int k = from; k < from + count; ++k) {
                    const int n = k >> 4, i = k & 15;
                    tot[other][n][i] = fmaf(fold, (float)acc[other][n][i], tot[other][n][i]);
                }
            };
            // Only the operands differ by kind; where there are no codes they are zeros.
            const int kind = now[f].kind;
            i32x4 w[S];
            if (kind == 6) raw[f].template operands<6>(w);
            else if (kind == 4) raw[f].template operands<4>(w);
            else if (kind == 2) raw[f].template operands<2>(w);
            else if (kind == 1) raw[f].template operands<1>(w);
            else {
#pragma unroll
                for (int s = 0; s < S; ++s) w[s] = i32x4{};
                if (kind == 0) {
                    const int terms = w_f32 ? 3 : 1;
                    const uint4* const wv = reinterpret_cast<const uint4*>(now[f].fields) + lane;
#pragma unroll 1
                    for (int term = 0; term < terms; ++term)
#pragma unroll
                        for (int s = 0; s < S; ++s)
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                const bf16x8 v = as_bf16x8(wv[((s * terms + term) * 2 + half) * 64]);
#pragma unroll
                                for (int n = 0; n < 2; ++n)
                                    tot[f][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(half == 0 ? eight_as_bf16(x[s][n].x, x[s][n].y) : eight_as_bf16(x[s][n].z, x[s][n].w), v, tot[f][n], 0, 0, 0);
                                __builtin_amdgcn_sched_barrier(0);
                            }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int s = 0; s < S; ++s) {
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    acc[f][n] = __builtin_amdgcn_mfma_i32_32x32x32_i8(as_i32x4(x[s][n]), w[s], s == 0 ? i32x16{} : acc[f][n], 0, 0, 0);
                    add_up((2 * s + n) * 16 / S, (2 * s + n + 1) * 16 / S - (2 * s + n) * 16 / S);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (both) {
#pragma unroll
                for (int n = 0; n < 2; ++n) tot[f][n] = __builtin_amdgcn_mfma_f32_32x32x2f32(pair_sum[n], pair_beta[f], tot[f][n], 0, 0, 0);
            }
        };
        phase(Const<0>());
        phase(Const<1>());
        behind = alpha[1];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            now[f] = unit_of(f, then);
            raw[f].load(now[f].kind, now[f].fields, lane);
            const float v = affine[f][(then / Q.per_chunk) * 64];
            alpha[f] = now[f].kind == 0 || now[f].kind == 7 ? 0.0f : v;
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) tot[1][n][i] = fmaf(behind, (float)acc[1][n][i], tot[1][n][i]);

    YT* __restrict__ const Y = static_cast<YT*>(Q.Y);
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t t = t0 + wt * 64 + n * 32 + g * 8 + hh * 4 + i;
                if (t >= Q.T) continue;
                const float scale = Q.scale[t];
#pragma unroll
                for (int f = 0; f < (PAIR ? 1 : 2); ++f) {
                    const int64_t lrow = in[f] * EIGHT_ROWS + sub;
                    if (b[f] >= Q.NB || lrow >= Q.R_u) continue;
                    float v = tot[f][n][g * 4 + i] * scale;
                    if constexpr (PAIR) {
                        float none;
                        v = activation<false>(Q.act, v, none) * (tot[1][n][g * 4 + i] * scale);
                    }
                    eight_store(Y + t * Q.ldy + rb[f] * Q.R_u + lrow, v);
                }
            }
}

#endif  // __HIPCC__

}  // namespace windq
