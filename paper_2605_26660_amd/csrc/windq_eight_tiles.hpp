// Products of many 8-bit tokens with a plan laid out for them: tiles of 64 WR rows x 64 tokens (of a pair: 32 WR rows of both).
#pragma once

#include "windq_eight.hpp"

namespace windq {

#ifdef __HIPCC__

template <int V>
struct Const {
    static constexpr int value = V;
};

template <typename YT, int S, int WR, bool PAIR>
__global__ __launch_bounds__(WR * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void eight_tiles_kernel(const EightArgs Q, const uint32_t row_tiles) {
    constexpr int TOKENS = 64, LOADS = 8 / WR;
    constexpr int SUMS = 64;                                // k-blocks whose words are in registers, a lane each, and whose tokens' sums are in LDS
    __shared__ uint4 xt[3][2][TOKENS * 8];
    __shared__ int32_t st[TOKENS * (SUMS + 1)];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, sub = lane & 31, hh = lane >> 5;
    const bool w_f32 = Q.w_f32 != 0;
    // Consecutive workgroups land on the eight XCDs in turn; each XCD gets a run of tiles that share tokens.
    const uint32_t n_tiles = gridDim.x, per = n_tiles >> 3;
    const uint32_t tile = blockIdx.x < per * 8 ? (blockIdx.x & 7) * per + (blockIdx.x >> 3) : blockIdx.x;
    const uint32_t tb = tile / row_tiles;
    const int64_t b0 = (int64_t)(tile - tb * row_tiles) * WR + wave, t0 = (int64_t)tb * TOKENS;
    const int32_t n_kb = Q.n_kb;

    // a wavefront's two row blocks: neighbours, or the same of the gate and of the up; past the last one: computed for nothing, stored by nobody
    int64_t b[2], rb[2], in[2];
    const uint32_t* words[2];
    const float* affine[2];
#pragma unroll
    for (int f = 0; f < 2; ++f) {
        b[f] = PAIR ? b0 : 2 * b0 + f;
        const int64_t at = b[f] < Q.NB ? b[f] : Q.NB - 1;
        rb[f] = at / Q.RB;
        in[f] = at - rb[f] * Q.RB;
        const char* const image = Q.P[PAIR ? f : 0].image;
        words[f] = reinterpret_cast<const uint32_t*>(image) + at * n_kb;
        affine[f] = reinterpret_cast<const float*>(image + Q.affine) + at * n_kb * 64 + sub;
    }

    // X: a row of 128 bytes a token, eight slots; slot p of token n holds slot p ^ (n / 2 & 7)
    const int8_t* xsrc[LOADS];
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
        const int n = (k * WR + wave) * 8 + (lane >> 3), slot = (lane & 7) ^ ((n >> 1) & 7);
        const int64_t t = t0 + n < Q.T ? t0 + n : Q.T - 1;
        xsrc[k] = Q.codes + t * Q.width + (slot < 2 * S ? slot : 0) * 16;
    }
    const uint32_t lds_xt = lds_address(xt);
    auto load_x = [&](int32_t pair, int stage) {            // past the last one: the last one again
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int32_t kb = 2 * pair + q < n_kb ? 2 * pair + q : n_kb - 1;
#pragma unroll
            for (int k = 0; k < LOADS; ++k)
                lds_load16(lds_xt + ((stage * 2 + q) * (TOKENS * 8) + (k * WR + wave) * 64) * 16, xsrc[k] + (int64_t)kb * (32 * S));
        }
    };
    const uint32_t lds_st = lds_address(st);
    auto load_sums = [&](int32_t kb) {
#pragma unroll 1
        for (int n = wave; n < TOKENS; n += WR)
            lds_load4(lds_st + n * (SUMS + 1) * 4, Q.sums + (t0 + n < Q.T ? t0 + n : Q.T - 1) * Q.sums_ld + (kb + lane < n_kb ? kb + lane : n_kb - 1));
    };

    // The words of SUMS k-blocks, checked; those of the next ones are on their way meanwhile.
    auto load_words = [&](int f, int32_t kb) {
        const int32_t at = kb + lane;
        return at < n_kb ? eight_word(Q.P[PAIR ? f : 0], words[f][at], S, w_f32) : (uint32_t)EIGHT_NOTHING;
    };
    auto block_of = [&](int f, uint32_t of, int32_t kb) {
        return eight_block(Q.P[PAIR ? f : 0], (uint32_t)__builtin_amdgcn_readlane((int)of, kb & (SUMS - 1)));
    };

    f32x16 tot[2][2] = {};
    i32x16 acc[2][2] = {};
    EightFields<S> raw[2];
    EightBlock now[2], next[2];
    uint32_t word[2], word_next[2];
    float alpha[2], alpha_next[2], behind = 0.0f;           // of the k-block; of the second row block's sums that are still to be added up
    float beta[2];                                          // of a pair of k-blocks, a lane's half one of them
    auto load_beta = [&](int32_t pair) {
        const int32_t kb = 2 * pair + hh < n_kb ? 2 * pair + hh : n_kb - 1;
#pragma unroll
        for (int f = 0; f < 2; ++f) beta[f] = affine[f][(int64_t)kb * 64 + 32];
    };
    const char* const xb = reinterpret_cast<const char*>(xt) + sub * 128;
    uint4 x[S][2];
    auto read_x = [&](int s, int half) {
#pragma unroll
        for (int n = 0; n < 2; ++n) x[s][n] = *reinterpret_cast<const uint4*>(xb + half * (TOKENS * 128) + n * 32 * 128 + (((2 * s + hh) ^ ((sub >> 1) & 7)) << 4));
    };
    const int32_t n_pairs = (n_kb + 1) >> 1;
    load_x(0, 0);
    load_sums(0);
#pragma unroll
    for (int f = 0; f < 2; ++f) word[f] = load_words(f, 0);
    load_x(1, 1);
    load_beta(0);
#pragma unroll
    for (int f = 0; f < 2; ++f) {
        word_next[f] = load_words(f, SUMS);
        now[f] = block_of(f, word[f], 0);
        raw[f].load(now[f].kind, now[f].fields, lane);
        alpha[f] = affine[f][0];
    }
    wait_for_loads();
    __syncthreads();
#pragma unroll
    for (int s = 0; s < S; ++s) read_x(s, 0);

    // Pairs of k-blocks.  Tokens are asked for two pairs ahead, and read into registers while the k-block before is multiplied: a stage that is
    // written to has been read by everybody a barrier ago.
    int stage = 0;
    for (int32_t pair = 0; pair < n_pairs; ++pair) {
        wait_for_loads();
        __syncthreads();
        if (pair != 0 && (pair & (SUMS / 2 - 1)) == 0) {    // the next sums, this pair's among them
            load_sums(2 * pair);
#pragma unroll
            for (int f = 0; f < 2; ++f) word_next[f] = load_words(f, 2 * pair + SUMS);
            wait_for_loads();
            __syncthreads();
        }
        const int stage1 = stage == 2 ? 0 : stage + 1, stage2 = stage1 == 2 ? 0 : stage1 + 1;
        load_x(pair + 2, stage2);
        float pair_beta[2], pair_sum[2];
#pragma unroll
        for (int f = 0; f < 2; ++f) pair_beta[f] = 2 * pair + hh < n_kb ? beta[f] : 0.0f;
#pragma unroll
        for (int n = 0; n < 2; ++n) pair_sum[n] = (float)st[(n * 32 + sub) * (SUMS + 1) + ((2 * pair + hh) & (SUMS - 1))];
        load_beta(pair + 1);

        auto k_block = [&](auto HALF) {
            constexpr int half = decltype(HALF)::value;
            const int32_t then = 2 * pair + half + 1;
            if (half == 1 && (then & (SUMS - 1)) == 0) {
#pragma unroll
                for (int f = 0; f < 2; ++f) word[f] = word_next[f];
            }
#pragma unroll
            for (int f = 0; f < 2; ++f) next[f] = block_of(f, word[f], then);
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
                raw[f].operands(kind, w);
                __builtin_amdgcn_sched_barrier(0);
                raw[f].load(next[f].kind, next[f].fields, lane);
                alpha_next[f] = affine[f][(int64_t)(then < n_kb ? then : n_kb - 1) * 64];
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int s = 0; s < S; ++s) {
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        acc[f][n] = __builtin_amdgcn_mfma_i32_32x32x32_i8(as_i32x4(x[s][n]), w[s], s == 0 ? i32x16{} : acc[f][n], 0, 0, 0);
                        add_up((2 * s + n) * 16 / S, (2 * s + n + 1) * 16 / S - (2 * s + n) * 16 / S);
                        if (f == 1 && n == 1) read_x(s, half == 0 ? 2 * stage + 1 : 2 * stage1);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                asm volatile("" : "+v"(tot[other][0]), "+v"(tot[other][1]));       // here, between the matrix instructions, and not in a later block
                if (half == 1) {                            // beta times the tokens' sums, two k-blocks an instruction
#pragma unroll
                    for (int n = 0; n < 2; ++n) tot[f][n] = __builtin_amdgcn_mfma_f32_32x32x2f32(pair_sum[n], pair_beta[f], tot[f][n], 0, 0, 0);
                }
            };
            phase(Const<0>());
            phase(Const<1>());
            behind = alpha[1];
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                now[f] = next[f];
                alpha[f] = alpha_next[f];
            }
        };
        k_block(Const<0>());
        k_block(Const<1>());
        stage = stage1;
    }
    wait_for_loads();
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) tot[1][n][i] = fmaf(behind, (float)acc[1][n][i], tot[1][n][i]);

    // Weights that stay as they are, with the tokens from where they lie: few k-blocks, and no others wait for them.  All of a k-block's loads are
    // asked for at once.
    for (int32_t kb0 = 0; kb0 < n_kb; kb0 += 64) {
        uint32_t of[2];
        uint64_t kept[2];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            of[f] = load_words(f, kb0);
            kept[f] = __ballot((of[f] & 7u) == 0u);
        }
        for (uint64_t left = kept[0] | kept[1]; left != 0; left &= left - 1) {
            const int at = __builtin_ctzll(left);
            uint4 v[2][S];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const int64_t t = t0 + n * 32 + sub;
                const int8_t* const from = Q.codes + (t < Q.T ? t : Q.T - 1) * Q.width + (int64_t)(kb0 + at) * (32 * S) + hh * 16;
#pragma unroll
                for (int s = 0; s < S; ++s) v[n][s] = *reinterpret_cast<const uint4*>(from + s * 32);
            }
            const int terms = w_f32 ? 3 : 1;
#pragma unroll 1
            for (int term = 0; term < terms; ++term) {
                uint4 w[2][S][2] = {};
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    if (((kept[f] >> at) & 1ull) == 0) continue;
                    const uint4* const from = reinterpret_cast<const uint4*>(block_of(f, of[f], at).fields) + lane;
#pragma unroll
                    for (int s = 0; s < S; ++s)
#pragma unroll
                        for (int half = 0; half < 2; ++half) w[f][s][half] = from[((s * terms + term) * 2 + half) * 64];
                }
#pragma unroll
                for (int s = 0; s < S; ++s)
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int n = 0; n < 2; ++n) {
                            const bf16x8 xv = half == 0 ? eight_as_bf16(v[n][s].x, v[n][s].y) : eight_as_bf16(v[n][s].z, v[n][s].w);
#pragma unroll
                            for (int f = 0; f < 2; ++f) tot[f][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xv, as_bf16x8(w[f][s][half]), tot[f][n], 0, 0, 0);
                        }
            }
        }
    }

    float scale[2][16];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int64_t t = t0 + n * 32 + (i >> 2) * 8 + hh * 4 + (i & 3);
            scale[n][i] = Q.scale[t < Q.T ? t : Q.T - 1];
        }
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            tot[0][n][i] *= scale[n][i];
            tot[1][n][i] *= scale[n][i];
            if constexpr (PAIR) {
                float none;
                tot[0][n][i] = activation<false>(Q.act, tot[0][n][i], none) * tot[1][n][i];
            }
        }
#pragma unroll
    for (int f = 0; f < (PAIR ? 1 : 2); ++f) {
        const int64_t lrow = in[f] * EIGHT_ROWS + sub;
        if (b[f] >= Q.NB || lrow >= Q.R_u) continue;
        const int64_t t1 = t0 + hh * 4;
        YT* __restrict__ const y = static_cast<YT*>(Q.Y) + t1 * Q.ldy + rb[f] * Q.R_u + lrow;
        if (t0 + TOKENS <= Q.T) {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) eight_store(y + (n * 32 + (i >> 2) * 8 + (i & 3)) * Q.ldy, tot[f][n][i]);
        } else {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int at = n * 32 + (i >> 2) * 8 + (i & 3);
                    if (t1 + at < Q.T) eight_store(y + at * Q.ldy, tot[f][n][i]);
                }
        }
    }
}

#endif  // __HIPCC__

}  // namespace windq
