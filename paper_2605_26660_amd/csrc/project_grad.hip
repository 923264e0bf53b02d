// windq_project_grad: the way back of a packed product with adapters beside it.
//   dh_t = alpha_k B_k^T dY_t     dX[t] = w_hat^T dY_t + A_k^T dh_t     dA[k] = sum_t dh_t x_t^T     dB[k] = alpha_k sum_t dY_t h_t^T
#include <math.h>

#include "windq_gemm.hpp"

namespace windq {

int check_tokens(const windq_mat* M, int64_t width, bool vector);

// ------------------------------------------------------------------------------------------------ layouts
// out [n][C][ldo] = in [n][R][C] transposed, rows padded with zeros up to ldo.
template <typename T>
__device__ __forceinline__ void transpose(const T* __restrict__ in, int64_t R, int32_t C, int64_t ldo, T* __restrict__ out, int64_t block) {
    __shared__ T tile[64][65];
    const int64_t rt = (ldo + 63) / 64, ct = (C + 63) / 64;
    const int64_t k = block / (rt * ct), rest = block - k * rt * ct;
    const int64_t r0 = rest / ct * 64, c0 = (rest - rest / ct * ct) * 64;
    for (int i = threadIdx.x; i < 4096; i += 256) {
        const int64_t r = r0 + (i >> 6), c = c0 + (i & 63);
        tile[i >> 6][i & 63] = r < R && c < C ? in[(k * R + r) * C + c] : (T)0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 4096; i += 256) {
        const int64_t c = c0 + (i >> 6), r = r0 + (i & 63);
        if (c < C && r < ldo) out[(k * C + c) * ldo + r] = tile[i & 63][i >> 6];
    }
}

inline int64_t transpose_workgroups(int64_t n, int64_t C, int64_t ldo) { return n * ((ldo + 63) / 64) * ((C + 63) / 64); }

// A copy of dY whose rows start on 16 bytes and end with zeros.
template <typename T>
__global__ __launch_bounds__(256) void align_kernel(const T* __restrict__ in, int64_t ld, int64_t T_, int64_t width, int64_t ldo, T* __restrict__ out, int64_t first) {
    const int64_t i = (first + blockIdx.x) * 256 + threadIdx.x;
    if (i >= T_ * ldo) return;
    const int64_t t = i / ldo, c = i - t * ldo;
    out[i] = c < width ? in[t * ld + c] : (T)0;
}

// ------------------------------------------------------------------------------------------------ dA and dB
// out = sum over an adapter's tokens of left_t right_t^T.  fp32: a lane owns a column of the right side and sixteen ranks, and has four tokens on
// their way at a time (bound by their latency: an adapter's tokens are few where calls are small).  Both sums in one launch.
struct OuterRows {
    const float* right;        // [T][ld]
    int64_t ld, width;
    const float* left;         // [T][max_rank]
    bool scaled, by_column;
    float* out;
};

__global__ __launch_bounds__(256) void outer_kernel(const OuterRows Q1, const OuterRows Q2, const int64_t first2, const AdapterArgs A, const GroupArgs G, const int64_t first) {
    const int64_t id = first + blockIdx.x;
    const OuterRows& Q = id < first2 ? Q1 : Q2;
    const int64_t block = id < first2 ? id : id - first2;
    const int64_t wt = (Q.width + 255) / 256;
    const int32_t groups = (A.max_rank + 15) / 16;
    const int32_t k = (int32_t)(block / (wt * groups));
    const int64_t rest = block - k * wt * groups;
    const int32_t r0 = (int32_t)(rest / wt) * 16;
    const int64_t c = (rest - rest / wt * wt) * 256 + threadIdx.x;
    if (c >= Q.width) return;
    const int32_t rank = adapter_rank(A, k), n = G.count[k], p0 = G.first[k];
    const int32_t ranks = A.max_rank - r0 < 16 ? A.max_rank - r0 : 16;
    float acc[16] = {};
    if (r0 < rank) {
        constexpr int AHEAD = 4;
        for (int32_t i0 = 0; i0 < n; i0 += AHEAD) {
            float x[AHEAD], l[AHEAD][16];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int64_t t = G.place[p0 + (i0 + i < n ? i0 + i : n - 1)];          // past the last token: read again, not counted
                x[i] = Q.right[t * Q.ld + c];
#pragma unroll
                for (int r = 0; r < 16; ++r) l[i][r] = Q.left[t * A.max_rank + r0 + (r < ranks ? r : 0)];
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (i0 + i < n) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[r] = fmaf(l[i][r], x[i], acc[r]);
                }
        }
    }
    const float factor = Q.scaled && A.alpha != nullptr ? A.alpha[k] : 1.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        if (r >= ranks) break;
        const float v = r0 + r < rank && n > 0 ? factor * acc[r] : 0.0f;
        if (Q.by_column) Q.out[((int64_t)k * Q.width + c) * A.max_rank + r0 + r] = v;
        else Q.out[((int64_t)k * A.max_rank + r0 + r) * Q.width + c] = v;
    }
}

// The same for bfloat16 on the matrix instructions: up to 64 ranks by 64 columns of the right side a wavefront, the sum over an adapter's places 32 at a
// time.  Eight wavefronts share the places (PARTS = 8, many tokens an adapter) or four pairs do, a pair's two with 64 columns each.  The sum runs over tokens, and an operand wants eight consecutive tokens of one column in a lane, while
// a token's columns lie side by side: a lane reads eight tokens by four columns and pairs tokens up in registers, which gives one
// operand for each of its four columns (every fourth column shares an instruction, as in the reconstruction).  The left side comes
// transposed and as three bfloat16 terms, so products are exact to fp32.  Bound by latency: a wavefront has a
// step's operands on their way while it multiplies the step before, and the tokens of the step after.
constexpr int OUTER_THREADS = 512;
inline int outer_parts(int64_t T, int32_t n) { return T >= (int64_t)512 * n ? 8 : 4; }        // 2048 tokens of one adapter: 35 to 42 us by eight, 81 by pairs; 700 of sixteen: 20 and 13
struct OuterArgs {
    const uint16_t* right;     // [T][ld], on 16 bytes, columns in eights readable
    int64_t ld, width;
    const uint16_t* planes;    // [3][max_rank][places]
    int64_t places;
    const int32_t* place;
    const int32_t* first;
    const int32_t* count;
    AdapterArgs A;
    bool scaled, by_column;
    float* out;
    int64_t tiles;             // of OUTER_COLS columns
};

template <int RF, int OUTER_PARTS>
__global__ __launch_bounds__(OUTER_THREADS) void outer_tiles_kernel(const OuterArgs Q1, const OuterArgs Q2, const int64_t first2, const int64_t first) {
    constexpr int OUTER_COLS = 512 / OUTER_PARTS;
    __shared__ float red[OUTER_PARTS / 2][RF * 16][OUTER_COLS + 4];
    const int64_t id = first + blockIdx.x;
    const OuterArgs& Q = id < first2 ? Q1 : Q2;
    const int64_t block = id < first2 ? id : id - first2;
    const int32_t groups = (Q.A.max_rank + 63) / 64;
    const int32_t k = (int32_t)(block / (Q.tiles * groups));
    const int64_t rest = block - k * Q.tiles * groups;
    const int32_t r0 = (int32_t)(rest / Q.tiles) * 64;
    const int64_t c0 = (rest - rest / Q.tiles * Q.tiles) * OUTER_COLS;
    const int part = (threadIdx.x >> 6) * OUTER_PARTS / 8, side = OUTER_PARTS == 8 ? 0 : ((threadIdx.x >> 6) & 1) * 64, lane = threadIdx.x & 63, sub = lane & 15, q = lane >> 4;
    const int32_t rank = adapter_rank(Q.A, k), n = Q.count[k], p0 = Q.first[k];
    const int64_t col = c0 + side + sub * 4;
    f32x4 acc[4][RF] = {};
    if (r0 < rank && n > 0) {
        // past the last token, and past the last column, what lies there is read again and counted as zeros
        const int64_t at_col = col < Q.width ? col : 0;
        auto places_of = [&](int32_t i0, int4 (&t)[2]) {
            const int32_t at = i0 + q * 8 < n ? i0 + q * 8 : 0;           // a slot's places are all written
            t[0] = *reinterpret_cast<const int4*>(Q.place + p0 + at);
            t[1] = *reinterpret_cast<const int4*>(Q.place + p0 + at + 4);
        };
        auto operands_of = [&](int32_t i0, const int4 (&p)[2], uint2 (&x)[8], uint4 (&b)[3][RF]) {
            const int32_t t[8] = {p[0].x, p[0].y, p[0].z, p[0].w, p[1].x, p[1].y, p[1].z, p[1].w};
            const int32_t at = i0 < n ? i0 : 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = *reinterpret_cast<const uint2*>(Q.right + (int64_t)(t[j] < 0 ? t[0] : t[j]) * Q.ld + at_col);
#pragma unroll
            for (int m = 0; m < 3; ++m)
#pragma unroll
                for (int f = 0; f < RF; ++f) {
                    const int32_t r = r0 + f * 16 + sub;
                    b[m][f] = *reinterpret_cast<const uint4*>(Q.planes + ((int64_t)m * Q.A.max_rank + (r < rank ? r : 0)) * Q.places + p0 + at + q * 8);
                }
        };
        uint2 x[8], next_x[8];
        uint4 b[3][RF], next_b[3][RF];
        int4 t[2];
        places_of(part * 32, t);
        operands_of(part * 32, t, x, b);
        places_of((part + OUTER_PARTS) * 32, t);
        for (int32_t i0 = part * 32; i0 < n; i0 += OUTER_PARTS * 32) {
            operands_of(i0 + OUTER_PARTS * 32, t, next_x, next_b);
            places_of(i0 + 2 * OUTER_PARTS * 32, t);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (i0 + q * 8 + j >= n || col >= Q.width) x[j] = make_uint2(0u, 0u);
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                uint32_t w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = m < 2 ? x[j].x : x[j].y;
                const uint32_t pick = (m & 1) != 0 ? 0x07060302u : 0x05040100u;         // halves of two tokens side by side
                const bf16x8 a = as_bf16x8(make_uint4(__builtin_amdgcn_perm(w[1], w[0], pick), __builtin_amdgcn_perm(w[3], w[2], pick),
                                                      __builtin_amdgcn_perm(w[5], w[4], pick), __builtin_amdgcn_perm(w[7], w[6], pick)));
#pragma unroll
                for (int f = 0; f < RF; ++f)
#pragma unroll
                    for (int p = 2; p >= 0; --p) acc[m][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, as_bf16x8(b[p][f]), acc[m][f], 0, 0, 0);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = next_x[j];
#pragma unroll
            for (int m = 0; m < 3; ++m)
#pragma unroll
                for (int f = 0; f < RF; ++f) b[m][f] = next_b[m][f];
        }
    }
    // the upper half of the parts hand theirs to the lower half, until one has all: a fixed order
#pragma unroll
    for (int round = OUTER_PARTS / 2; round >= 1; round >>= 1) {
        if (part >= round && part < 2 * round) {
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int f = 0; f < RF; ++f)
#pragma unroll
                    for (int i = 0; i < 4; ++i) red[part - round][f * 16 + sub][side + (4 * q + i) * 4 + m] = acc[m][f][i];
        }
        __syncthreads();
        if (part < round) {
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int f = 0; f < RF; ++f)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[m][f][i] += red[part][f * 16 + sub][side + (4 * q + i) * 4 + m];
        }
        __syncthreads();
    }
    if (part == 0) {
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int f = 0; f < RF; ++f)
#pragma unroll
                for (int i = 0; i < 4; ++i) red[0][f * 16 + sub][side + (4 * q + i) * 4 + m] = acc[m][f][i];
    }
    __syncthreads();
    const float factor = Q.scaled && Q.A.alpha != nullptr ? Q.A.alpha[k] : 1.0f;
    const int32_t R = Q.A.max_rank, ranks = R - r0 < RF * 16 ? R - r0 : RF * 16;
    const int64_t left = Q.width - c0;
    const int32_t cols = left < OUTER_COLS ? (int32_t)left : OUTER_COLS;
    for (int e = threadIdx.x; e < ranks * OUTER_COLS; e += OUTER_THREADS) {
        const int r = Q.by_column ? e % ranks : e / OUTER_COLS, c = Q.by_column ? e / ranks : e % OUTER_COLS;
        if (c >= cols) continue;
        const float v = r0 + r < rank && n > 0 ? factor * red[0][r][c] : 0.0f;
        if (Q.by_column) Q.out[((int64_t)k * Q.width + c0 + c) * R + r0 + r] = v;
        else Q.out[((int64_t)k * R + r0 + r) * Q.width + c0 + c] = v;
    }
}

// ------------------------------------------------------------------------------------------------ dX
struct DxArgs {
    PackArgs P;                // rows, cols alone where packed is false
    bool packed;
    const void* dY;            // rows on 16 bytes, readable up to a multiple of 8
    int64_t ldy;
    int64_t T;
    void* dX;
    int64_t ldx;
    const float* dh;           // [T][max_rank] or null
    AdapterArgs A;
    float* part;               // sums of parts of the rows; fp32: [splits][tiles][4][256][4], bfloat16: [splits][T][cols]
    int32_t splits;
};

// Eight columns of A_k^T dh_t, added to v.
__device__ __forceinline__ void add_adapter8(const AdapterArgs& A, const float* __restrict__ dh, int64_t t, int64_t col, int64_t cols, float (&v)[8]) {
    const int32_t k = A.of[t];
    if (k < 0 || k >= A.n) return;
    const int32_t rank = adapter_rank(A, k);
    const uint16_t* __restrict__ const a = static_cast<const uint16_t*>(A.a) + (int64_t)k * A.max_rank * cols + col;
    float sum[8] = {};
#pragma unroll 4
    for (int32_t r = 0; r < rank; ++r) {
        float av[8];
        load8(a + (int64_t)r * cols, av);
        const float d = dh[t * A.max_rank + r];
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = fmaf(av[j], d, sum[j]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += sum[j];
}

__device__ __forceinline__ void skip_row(const PackArgs& P, int64_t row, int64_t col, float (&w)[8]) {
    if (P.w_f32 != 0) load8(static_cast<const float*>(P.W) + row * P.ld + col, w);
    else load8(static_cast<const uint16_t*>(P.W) + row * P.ld + col, w);
}

// An octet of one row as fp32 weights (rounded nowhere but by the multiply-add).
__device__ __forceinline__ void weight_octet(const PackArgs& P, int64_t row, int64_t col, const uint16_t* __restrict__ trits_of, float (&w)[8]) {
    const int64_t rb = row / P.R_u, lrow = row - rb * P.R_u;
    const int32_t j = (int32_t)(col / P.G), o = (int32_t)(col - (int64_t)j * P.G) >> 3;
    const int64_t u = rb * P.n_chunks + j;
    int64_t base;
    const int a = pk_action(P, u, base);
    if (a == 0) return skip_row(P, row, col, w);
    const int64_t g = u * P.R_u + lrow;
    const float s = P.scale[g], of = a >= 5 ? 0.0f : P.offset[g];
    const uint4 f = octet_fields(a, P.codes + base + lrow * pk_bytes_per_group(a, P.G), o, trits_of);
    const float f0 = pk_f0(a);
    const uint32_t m = P.mask != nullptr ? P.mask[row * P.mask_ld + (col >> 3)] : 0u;
    const uint32_t v[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = ((i & 1) != 0 ? __uint_as_float(v[i >> 1] & 0xffff0000u) : bf16_bits_to_f32(v[i >> 1] & 0xffffu)) - f0;
        w[i] = ((m >> i) & 1u) != 0u ? 0.0f : fmaf(q, s, of);
    }
}

// bfloat16: the sums of the product's parts (none: the packed matrix is not wanted) and the adapters', a thread per token and octet of columns.
__global__ __launch_bounds__(256) void dx_join_kernel(const DxArgs Q, const int64_t first) {
    const int64_t i = (first + blockIdx.x) * 256 + threadIdx.x, octets = Q.P.cols >> 3;
    const int64_t t = i / octets, c = (i - t * octets) * 8;
    if (t >= Q.T) return;
    float v[8] = {};
#pragma unroll 4
    for (int32_t s = 0; s < Q.splits; ++s) {
        float p[8];
        load8(Q.part + (s * Q.T + t) * Q.P.cols + c, p);
#pragma unroll
        for (int m = 0; m < 8; ++m) v[m] += p[m];
    }
    if (Q.dh != nullptr) add_adapter8(Q.A, Q.dh, t, c, Q.P.cols, v);
    uint16_t* __restrict__ const o = static_cast<uint16_t*>(Q.dX) + t * Q.ldx + c;
    uint32_t w[8];
#pragma unroll
    for (int m = 0; m < 8; ++m) w[m] = f32_to_bf16_bits(v[m]);
    if ((Q.ldx & 7) == 0 && (reinterpret_cast<uintptr_t>(Q.dX) & 15) == 0) {
        *reinterpret_cast<uint4*>(o) = pack8(w);
    } else {
#pragma unroll
        for (int m = 0; m < 8; ++m) o[m] = (uint16_t)w[m];
    }
}

// w_hat rounded to bfloat16 and turned: wt [cols][K], zeros from the last row to K.  A thread has eight rows by eight columns.
__device__ __forceinline__ void turn(const PackArgs& P, int32_t K, uint16_t* __restrict__ wt, int64_t block) {
    __shared__ uint16_t trits_of[256];
    trits_of[threadIdx.x] = (uint16_t)trit_fields(threadIdx.x);
    __syncthreads();
    const int32_t row_blocks = (K + 255) / 256;
    const int64_t cb = block / row_blocks;
    const int64_t r0 = (block - cb * row_blocks) * 256 + (threadIdx.x & 31) * 8, col = cb * 64 + (threadIdx.x >> 5) * 8;
    if (col >= P.cols || r0 >= K) return;
    uint32_t v[8][4];
    const uint32_t R_u = (uint32_t)P.R_u, rb = (uint32_t)r0 / R_u, lrow = (uint32_t)r0 - rb * R_u;
    if (r0 + 8 <= P.rows && lrow + 8 <= R_u) {              // one unit's rows
        const uint32_t j = (uint32_t)col / (uint32_t)P.G;
        const int o = ((int)col - (int)j * P.G) >> 3;
        const int64_t u = (int64_t)rb * P.n_chunks + j;
        int64_t base;
        const int a = pk_action(P, u, base);
        if (a == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float w0[8], w1[8];
                skip_row(P, r0 + 2 * i, col, w0);
                skip_row(P, r0 + 2 * i + 1, col, w1);
#pragma unroll
                for (int m = 0; m < 8; ++m) v[m][i] = f32_to_bf16_bits(w0[m]) | f32_to_bf16_bits(w1[m]) << 16;
            }
        } else {
            const int32_t nb = (int32_t)pk_bytes_per_group(a, P.G);
            const uint8_t* const first = P.codes + base + (int64_t)lrow * nb;
            float sc[8], of[8];
            __builtin_memcpy(sc, P.scale + u * P.R_u + lrow, 32);
            __builtin_memcpy(of, P.offset + u * P.R_u + lrow, 32);
            uint4 f[8];
            auto rows = [&](auto octet) {
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = octet(first + i * nb);
            };
            switch (a) {
                case 1: rows([&](const uint8_t* p) { uint2 q; __builtin_memcpy(&q, p + o * 8, 8); return fields8(q.x, q.y); }); break;
                case 2: rows([&](const uint8_t* p) { uint32_t q; __builtin_memcpy(&q, p + o * 4, 4); return fields4(q); }); break;
                case 3: rows([&](const uint8_t* p) { return octet_fields(3, p, o, trits_of); }); break;
                case 4: rows([&](const uint8_t* p) { uint16_t q; __builtin_memcpy(&q, p + o * 2, 2); return fields2(q); }); break;
                case 5: rows([&](const uint8_t* p) { return fields2(octet_trits(p, o, trits_of) & 0xffffu); }); break;
                default: rows([&](const uint8_t* p) { return fields1(p[o]); }); break;
            }
            const float f0 = pk_f0(a);
            uint32_t m8[8] = {};
            if (P.mask != nullptr) {
#pragma unroll
                for (int i = 0; i < 8; ++i) m8[i] = P.mask[(r0 + i) * P.mask_ld + (col >> 3)];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int m = 0; m < 8; ++m) {
                    uint32_t w[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint4& g = f[2 * i + k];
                        const uint32_t pair = (m >> 1) == 0 ? g.x : ((m >> 1) == 1 ? g.y : ((m >> 1) == 2 ? g.z : g.w));
                        const float q = ((m & 1) != 0 ? __uint_as_float(pair & 0xffff0000u) : __uint_as_float(pair << 16)) - f0;
                        const float x = fmaf(q, sc[2 * i + k], a >= 5 ? 0.0f : of[2 * i + k]);
                        w[k] = f32_to_bf16_bits(((m8[2 * i + k] >> m) & 1u) != 0u ? 0.0f : x);
                    }
                    v[m][i] = w[0] | w[1] << 16;
                }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float w0[8] = {}, w1[8] = {};
            if (r0 + 2 * i < P.rows) weight_octet(P, r0 + 2 * i, col, trits_of, w0);
            if (r0 + 2 * i + 1 < P.rows) weight_octet(P, r0 + 2 * i + 1, col, trits_of, w1);
#pragma unroll
            for (int m = 0; m < 8; ++m) v[m][i] = f32_to_bf16_bits(w0[m]) | f32_to_bf16_bits(w1[m]) << 16;
        }
    }
#pragma unroll
    for (int m = 0; m < 8; ++m) *reinterpret_cast<uint4*>(wt + (col + m) * K + r0) = make_uint4(v[m][0], v[m][1], v[m][2], v[m][3]);
}

// What the later kernels read, in one launch: the reconstruction turned, B and A transposed, tokens by adapter.  Workgroups in that order.
// 11008 x 4096: 29 to 33 us, 92 MB written (3.2 to 2.8 TB/s).
template <typename XT>
struct PrepareArgs {
    PackArgs P;
    int32_t K;
    uint16_t* wt;
    const XT* b;
    XT* bt;
    const XT* a;
    XT* at;
    int64_t ld;                // of B transposed
    AdapterArgs A;
    GroupArgs G;
    int64_t turns, bs, as, groups;
};

template <typename XT>
__global__ __launch_bounds__(256) void grad_prepare_kernel(const PrepareArgs<XT> Q, const int64_t first) {
    int64_t block = first + blockIdx.x;
    if (block < Q.turns) return turn(Q.P, Q.K, Q.wt, block);
    block -= Q.turns;
    if (block < Q.bs) return transpose(Q.b, Q.P.rows, Q.A.max_rank, Q.ld, Q.bt, block);
    block -= Q.bs;
    if (block < Q.as) return transpose(Q.a, (int64_t)Q.A.max_rank, (int32_t)Q.P.cols, (int64_t)Q.A.max_rank, Q.at, block);
    group_adapter(Q.G, (int32_t)(block - Q.as));
}

// fp32: 64 columns and 64 tokens a workgroup on the fp32 matrix instructions.  Sixteen wavefronts, four to a quarter of the rows, which go
// through LDS 32 at a time, the next ones on their way meanwhile: small layers leave few workgroups, and a wavefront's time is latency.
// Where tiles are fewer than the CUs the rows are split further, over workgroups, whose sums another kernel joins in order: 1000 x 1056 at 77
// tokens (34 tiles of 8 steps) takes 60 us without the split and 17 + 5 with it (four parts of 2 steps).
constexpr int DXF_THREADS = 1024, DXF_PARTS = DXF_THREADS / 256, DXF_TILES = 256;
inline int64_t dxf_tiles(int64_t T, int64_t cols) { return tokens_in(cols, 64) * tokens_in(T, 64); }
inline int32_t dxf_splits(int64_t tiles, int64_t rows) {
    const int64_t steps = tokens_in(rows, 32 * DXF_PARTS), most = DXF_TILES / tiles < 1 ? 1 : DXF_TILES / tiles;
    const int64_t each = tokens_in(steps, most < steps ? most : steps);
    return (int32_t)tokens_in(steps, each);
}

// Four columns of a token: the adapter's part, and out.
__device__ __forceinline__ void dx_f32_store(const DxArgs& Q, int64_t t, int64_t c, float (&v)[4]) {
    const PackArgs& P = Q.P;
    if (t >= Q.T || c >= P.cols) return;                    // columns come in eights: four of them are in or out together
    if (Q.dh != nullptr) {
        const int32_t k = Q.A.of[t];
        if (k >= 0 && k < Q.A.n) {
            const int32_t rank = adapter_rank(Q.A, k);
            const float* __restrict__ const a = static_cast<const float*>(Q.A.a) + (int64_t)k * Q.A.max_rank * P.cols + c;
            float sum[4] = {};
#pragma unroll 4
            for (int32_t r = 0; r < rank; ++r) {
                const float4 av = *reinterpret_cast<const float4*>(a + (int64_t)r * P.cols);
                const float d = Q.dh[t * Q.A.max_rank + r];
                sum[0] = fmaf(av.x, d, sum[0]);
                sum[1] = fmaf(av.y, d, sum[1]);
                sum[2] = fmaf(av.z, d, sum[2]);
                sum[3] = fmaf(av.w, d, sum[3]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += sum[i];
        }
    }
    float* __restrict__ const o = static_cast<float*>(Q.dX) + t * Q.ldx + c;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = v[i];
}

__global__ __launch_bounds__(256) void dx_f32_join_kernel(const DxArgs Q, const int64_t tiles, const int64_t first) {
    const int64_t tile = (first + blockIdx.x) >> 2, col_blocks = (Q.P.cols + 63) / 64, tb = tile / col_blocks;
    const int n = (int)(first + blockIdx.x) & 3, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    float v[4] = {};
    for (int32_t s = 0; s < Q.splits; ++s) {
        const float4 p = reinterpret_cast<const float4*>(Q.part)[(s * tiles + tile) * 1024 + n * 256 + threadIdx.x];
        v[0] += p.x;
        v[1] += p.y;
        v[2] += p.z;
        v[3] += p.w;
    }
    dx_f32_store(Q, tb * 64 + n * 16 + (lane & 15), (tile - tb * col_blocks) * 64 + wave * 16 + 4 * (lane >> 4), v);
}

__global__ __launch_bounds__(DXF_THREADS) void dx_f32_kernel(const DxArgs Q, const int64_t first) {
    __shared__ float wts[DXF_PARTS][32][68], yts[DXF_PARTS][32][68];
    __shared__ uint16_t trits_of[256];
    if (threadIdx.x < 256) trits_of[threadIdx.x] = (uint16_t)trit_fields(threadIdx.x);
    __syncthreads();
    const PackArgs& P = Q.P;
    const int part = threadIdx.x >> 8, tid = threadIdx.x & 255, wave = tid >> 6, lane = tid & 63, sub = lane & 15, q = lane >> 4;
    float(&wt)[32][68] = wts[part];
    float(&yt)[32][68] = yts[part];
    const int64_t col_blocks = (P.cols + 63) / 64, tiles = col_blocks * ((Q.T + 63) / 64);
    const int64_t block = first + blockIdx.x, split = block / tiles, tile = block - split * tiles, tb = tile / col_blocks;
    const int64_t c0 = (tile - tb * col_blocks) * 64, t0 = tb * 64;
    const float* __restrict__ const dY = static_cast<const float*>(Q.dY);
    f32x4 acc[4] = {};
    if (Q.packed) {
        // steps of a quarter, the same for all of them: barriers are shared
        const int64_t blocks = (P.rows + 31) / 32, each = (blocks + DXF_PARTS * Q.splits - 1) / (DXF_PARTS * Q.splits), from = (split * DXF_PARTS + part) * each;
        const int r = tid >> 3, o = tid & 7, yr = tid & 31;
        float w[8], y[8];
        auto fetch = [&](int64_t block) {
            const int64_t r0 = block * 32;
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = 0.0f;
            if (r0 + r < P.rows && c0 + o * 8 < P.cols) weight_octet(P, r0 + r, c0 + o * 8, trits_of, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int64_t t = t0 + (tid >> 5) + 8 * j;
                y[j] = r0 + yr < P.rows && t < Q.T ? dY[t * Q.ldy + r0 + yr] : 0.0f;
            }
        };
        fetch(from);
        for (int64_t i = 0; i < each; ++i) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                wt[r][o * 8 + j] = w[j];
                yt[yr][(tid >> 5) + 8 * j] = y[j];
            }
            __syncthreads();
            // past its quarter a part multiplies zeros
            fetch(i + 1 < each ? from + i + 1 : blocks);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float a = wt[k * 4 + q][wave * 16 + sub];
#pragma unroll
                for (int n = 0; n < 4; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, yt[k * 4 + q][n * 16 + sub], acc[n], 0, 0, 0);
            }
        }
        __syncthreads();
        // the parts' sums, in order
        float(*const red)[DXF_PARTS][4][64][4] = reinterpret_cast<float(*)[DXF_PARTS][4][64][4]>(&wts[0][0][0]);    // [n pair][part][wave][lane][i], two at a time
        static_assert(sizeof(float) * 2 * DXF_PARTS * 4 * 64 * 4 <= sizeof(wts), "the sums fit");
#pragma unroll
        for (int n2 = 0; n2 < 4; n2 += 2) {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) red[n][part][wave][lane][i] = acc[n2 + n][i];
            __syncthreads();
            if (part == 0) {
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float v = red[n][0][wave][lane][i];
#pragma unroll
                        for (int p = 1; p < DXF_PARTS; ++p) v += red[n][p][wave][lane][i];
                        acc[n2 + n][i] = v;
                    }
            }
            __syncthreads();
        }
    }
    if (part != 0) return;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        float v[4] = {acc[n][0], acc[n][1], acc[n][2], acc[n][3]};
        if (Q.splits > 1) reinterpret_cast<float4*>(Q.part)[block * 1024 + n * 256 + tid] = make_float4(v[0], v[1], v[2], v[3]);
        else dx_f32_store(Q, t0 + n * 16 + sub, c0 + wave * 16 + 4 * q, v);
    }
}

// ------------------------------------------------------------------------------------------------ the call
struct GradWs {
    size_t h, dh, bt, at, dy, place, owner, first, count, part, part2, planes_h, planes_dh, wt, gm, dxf, total;
    int64_t ld;                // of dY's copy and of B transposed
};

GradWs grad_ws(int32_t dtype, int64_t T, int64_t rows, int64_t cols, int32_t n, int32_t max_rank) {
    const size_t eb = dtype == WINDQ_F32 ? 4 : 2;
    const bool bf = dtype == WINDQ_BF16;
    GradWs w;
    w.ld = bf ? gemm_k(rows) : in_eights(rows);
    size_t at = 0;
    auto take = [&at](size_t bytes) {
        const size_t here = at;
        at += round_up(bytes, 256);
        return here;
    };
    const int64_t slots = group_slots(T, n);
    w.dy = take((size_t)(T * w.ld) * eb);
    w.h = take((size_t)(T * max_rank) * 4);
    w.dh = take((size_t)(T * max_rank) * 4);
    w.bt = take((size_t)n * (size_t)max_rank * (size_t)w.ld * eb);
    w.at = take(bf ? (size_t)n * (size_t)max_rank * (size_t)cols * eb : 0);
    w.place = take((size_t)slots * GROUP * 4);
    w.owner = take((size_t)slots * 4);
    w.first = take((size_t)n * 4);
    w.count = take((size_t)n * 4);
    w.part = take(bf && n > 0 ? shrink_floats(slots, in_eights(rows), max_rank) * 4 : 0);        // dh's pieces
    w.part2 = take(bf && n > 0 ? shrink_floats(slots, cols, max_rank) * 4 : 0);                  // h's
    w.planes_h = take(bf && n > 0 ? (size_t)slots * GROUP * (size_t)max_rank * 6 : 0);
    w.planes_dh = take(bf && n > 0 ? (size_t)slots * GROUP * (size_t)max_rank * 6 : 0);
    w.wt = take(bf && T > 0 ? (size_t)gemm_cols(cols) * (size_t)gemm_k(rows) * 2 : 0);
    w.gm = take(bf ? (size_t)gemm_parts(T, gemm_k(rows), cols) * 4 : 0);
    w.dxf = take(bf ? 0 : (size_t)DXF_TILES * 64 * 64 * 4);       // tiles x splits are no more
    w.total = at == 0 ? 256 : at;
    return w;
}

size_t grad_ws_bytes(int32_t dtype, int64_t T, int64_t rows, int64_t cols, int32_t n, int32_t max_rank) {
    return grad_ws(dtype, T, rows, cols, n, max_rank).total;
}

// Behind its arguments a kernel takes the first of a piece's workgroups.
#define WINDQ_LAUNCH(wgs, threads, kernel, ...)                                                                                                  \
    do {                                                                                                                                         \
        const int launched_ = launch_pieces(wgs, threads, [&](int64_t first_, dim3 g_) { kernel<<<g_, dim3(threads), 0, st>>>(__VA_ARGS__, first_); }); \
        if (launched_ != WINDQ_OK) return launched_;                                                                                             \
    } while (0)

template <typename XT>
int grad_all(DxArgs& Q, const windq_mat* dY, const windq_mat* X, const float* h, float* dA, float* dB, char* ws, const GradWs& at, hipStream_t st) {
    const int64_t T = Q.T, rows = Q.P.rows, cols = Q.P.cols;
    const bool side = Q.A.n > 0;
    constexpr bool bf = sizeof(XT) == 2;
    const bool turn = bf && Q.packed && Q.dX != nullptr && T > 0;
    const AdapterArgs A = Q.A;
    if (T > 0 && (dY->ld % 8 != 0 || rows % (turn ? GM_K : 8) != 0 || !aligned(dY->data, 16))) {
        XT* to = reinterpret_cast<XT*>(ws + at.dy);
        WINDQ_LAUNCH((T * at.ld + 255) / 256, 256, align_kernel<XT>, static_cast<const XT*>(dY->data), dY->ld, T, rows, at.ld, to);
        Q.dY = to;
        Q.ldy = at.ld;
    } else {
        Q.dY = dY->data;
        Q.ldy = dY->ld;
    }
    const XT* const dYv = static_cast<const XT*>(Q.dY);
    const int32_t rows8 = (int32_t)in_eights(rows);
    PrepareArgs<XT> R = {};
    R.P = Q.P;
    R.A = A;
    const GroupArgs G = {A.of, T, A.n, group_slots(T, A.n), reinterpret_cast<int32_t*>(ws + at.place), reinterpret_cast<int32_t*>(ws + at.owner),
                         reinterpret_cast<int32_t*>(ws + at.first), reinterpret_cast<int32_t*>(ws + at.count)};
    XT* const bt = reinterpret_cast<XT*>(ws + at.bt);
    const bool outer = dA != nullptr;
    if (turn) {
        R.K = (int32_t)gemm_k(rows);
        R.wt = reinterpret_cast<uint16_t*>(ws + at.wt);
        R.turns = ((cols + 63) / 64) * ((R.K + 255) / 256);
    }
    if (side) {
        R.b = static_cast<const XT*>(A.b);
        R.bt = bt;
        R.ld = at.ld;
        R.bs = transpose_workgroups(A.n, A.max_rank, at.ld);
        if (turn) {
            R.a = static_cast<const XT*>(A.a);
            R.at = reinterpret_cast<XT*>(ws + at.at);
            R.as = transpose_workgroups(A.n, cols, A.max_rank);
        }
        if (bf || outer) {
            R.G = G;
            R.groups = A.n;
        }
    }
    WINDQ_LAUNCH(R.turns + R.bs + R.as + R.groups, 256, grad_prepare_kernel<XT>, R);
    if (side) {
        float* const dh = reinterpret_cast<float*>(ws + at.dh);
        if constexpr (bf) {
            float* const part = reinterpret_cast<float*>(ws + at.part);
            uint16_t* const planes_h = reinterpret_cast<uint16_t*>(ws + at.planes_h);
            uint16_t* const planes_dh = reinterpret_cast<uint16_t*>(ws + at.planes_dh);
            float* const part2 = reinterpret_cast<float*>(ws + at.part2);
            auto pieces = [&](const void* x, int64_t ld, const void* a, int64_t lda, int64_t width, float* to) {
                return ShrinkArgs{x, ld, a, lda, (int32_t)width, shrink_splits(G.slots, width), G.slots, G.place, G.owner, A, to};
            };
            const ShrinkArgs S1 = pieces(Q.dY, Q.ldy, bt, at.ld, rows8, part);
            const JoinArgs J1 = {part, S1.splits, G.slots, G.place, G.owner, T, A, true, dh, outer ? planes_dh : nullptr, nullptr};
            JoinArgs J2 = {part2, 0, G.slots, G.place, G.owner, T, A, false, nullptr, planes_h, h};
            int status;
            if (outer && h == nullptr) {
                const ShrinkArgs S2 = pieces(X->data, X->ld, A.a, cols, cols, part2);
                J2.splits = S2.splits;
                status = launch_shrink(S1, &S2, st);
            } else {
                status = launch_shrink(S1, nullptr, st);
            }
            if (status == WINDQ_OK) status = launch_join(J1, outer ? &J2 : nullptr, st);
            if (status != WINDQ_OK) return status;
            if (outer) {
                const int32_t groups = (A.max_rank + 63) / 64;
                const int parts = outer_parts(T, A.n);
                const int64_t by = 512 / parts;
                OuterArgs O1 = {static_cast<const uint16_t*>(X->data), X->ld, cols, planes_dh, G.slots * GROUP, G.place, G.first, G.count, A, false, false, dA, tokens_in(cols, by)};
                OuterArgs O2 = {dYv, Q.ldy, rows, planes_h, G.slots * GROUP, G.place, G.first, G.count, A, true, true, dB, tokens_in(rows, by)};
                const int64_t n1 = (int64_t)A.n * groups * O1.tiles, n2 = (int64_t)A.n * groups * O2.tiles;
                const int32_t RF = A.max_rank >= 64 ? 4 : shrink_ranks(A.max_rank) / 16;
#define WINDQ_OUTER(F)                                                                                    \
    do {                                                                                                  \
        if (parts == 8) WINDQ_LAUNCH(n1 + n2, OUTER_THREADS, (outer_tiles_kernel<F, 8>), O1, O2, n1);     \
        else WINDQ_LAUNCH(n1 + n2, OUTER_THREADS, (outer_tiles_kernel<F, 4>), O1, O2, n1);                \
    } while (0)
                if (RF == 1) WINDQ_OUTER(1);
                else if (RF == 2) WINDQ_OUTER(2);
                else if (RF == 3) WINDQ_OUTER(3);
                else WINDQ_OUTER(4);
#undef WINDQ_OUTER
            }
        } else {
            AdapterArgs B = A;
            B.a = bt;
            int status = launch_shrink_token(dYv, Q.ldy, T, rows8, B, true, dh, st);
            if (status != WINDQ_OK) return status;
            if (outer) {
                if (h == nullptr) {
                    float* const ht = reinterpret_cast<float*>(ws + at.h);
                    status = launch_shrink_token(static_cast<const XT*>(X->data), X->ld, T, (int32_t)cols, A, false, ht, st);
                    if (status != WINDQ_OK) return status;
                    h = ht;
                }
                const int64_t groups = (int64_t)A.n * ((A.max_rank + 15) / 16);
                const OuterRows O1 = {static_cast<const float*>(X->data), X->ld, cols, dh, false, false, dA};
                const OuterRows O2 = {dYv, Q.ldy, rows, h, true, true, dB};
                const int64_t n1 = groups * tokens_in(cols, 256), n2 = groups * tokens_in(rows, 256);
                WINDQ_LAUNCH(n1 + n2, 256, outer_kernel, O1, O2, n1, A, G);
            }
        }
        Q.dh = dh;
    }
    if (Q.dX == nullptr || T == 0) return WINDQ_OK;
    if constexpr (bf) {
        if (turn) {
            // tiles are no more than 2^31 / 128^2 and two sides' edges: one launch holds them
            const int64_t tall = tokens_in(T, GM_N), by = tokens_in(cols, 256) * tall >= GM_TILES ? 256 : 128, tiles = tokens_in(cols, by) * tall;
            GemmArgs M = {R.wt, dYv, Q.ldy, R.K, T, cols, static_cast<uint16_t*>(Q.dX), Q.ldx, Q.dh, R.at, A, (uint32_t)tokens_in(cols, by), nullptr, (int32_t)tiles, R.K / GM_K};
            if (by == 256) {
                dx_gemm_kernel<4><<<dim3((uint32_t)tiles), dim3(GM_THREADS), 0, st>>>(M);
                return hipGetLastError() == hipSuccess ? WINDQ_OK : WINDQ_EHIP;
            }
            const int32_t each = gemm_each(R.K, tiles), splits = (int32_t)tokens_in(R.K / GM_K, each);
            if (splits > 1) {
                M.each = each;
                M.part = Q.part = reinterpret_cast<float*>(ws + at.gm);
                Q.splits = splits;
            }
            dx_gemm_kernel<2><<<dim3((uint32_t)(tiles * splits)), dim3(GM_THREADS), 0, st>>>(M);
            if (hipGetLastError() != hipSuccess) return WINDQ_EHIP;
            if (splits == 1) return WINDQ_OK;
        }
        WINDQ_LAUNCH(tokens_in(T * (cols / 8), 256), 256, dx_join_kernel, Q);
    } else {
        const int64_t tiles = dxf_tiles(T, cols);
        Q.splits = Q.packed ? dxf_splits(tiles, rows) : 1;
        Q.part = reinterpret_cast<float*>(ws + at.dxf);
        WINDQ_LAUNCH(tiles * Q.splits, DXF_THREADS, dx_f32_kernel, Q);
        if (Q.splits > 1) WINDQ_LAUNCH(tiles * 4, 256, dx_f32_join_kernel, Q, tiles);
    }
    return WINDQ_OK;
}

}  // namespace windq

using namespace windq;

extern "C" int windq_project_grad(const windq_packed* P, const windq_mat* dY, const windq_mat* X, const windq_adapters* adapters,
                                  const int32_t* adapter_of, const float* h, void* dX, int64_t ld_dx, float* dA, float* dB, void* ws,
                                  size_t ws_bytes, void* stream) {
    DxArgs Q = {};
    Q.packed = P != nullptr;
    int status;
    if (P != nullptr) {
        status = check_packed(P, &Q.P);
        if (status != WINDQ_OK) return status;
    } else {
        if (dY == nullptr || X == nullptr || adapters == nullptr) return WINDQ_EINVAL;
        Q.P.rows = dY->cols;
        Q.P.cols = X->cols;
        if (Q.P.rows <= 0 || Q.P.cols <= 0 || Q.P.cols % 8 != 0 || Q.P.rows > (int64_t)1 << 31 || Q.P.cols > (int64_t)1 << 31) return WINDQ_ESHAPE;
    }
    status = check_tokens(dY, Q.P.rows, false);
    if (status != WINDQ_OK) return status;
    const int64_t T = dY->rows;
    if (!grad_sizes_fit(T, Q.P.rows, Q.P.cols)) return WINDQ_ESHAPE;
    if ((dA == nullptr) != (dB == nullptr)) return WINDQ_EINVAL;
    if (adapters != nullptr) {
        static const int32_t nobody = -1;
        status = check_adapters(adapters, T == 0 ? &nobody : adapter_of, dY->dtype, &Q.A);
        if (status != WINDQ_OK) return status;
        if (dA != nullptr) {
            status = check_tokens(X, Q.P.cols, true);
            if (status != WINDQ_OK) return status;
            if (X->dtype != dY->dtype) return WINDQ_EDTYPE;
            if (X->rows != T) return WINDQ_ESHAPE;
            if (!aligned(dA, 16) || !aligned(dB, 16) || !aligned(h, 16)) return WINDQ_EINVAL;
        }
    } else if (dA != nullptr) {
        return WINDQ_EINVAL;
    }
    if (dX == nullptr && dA == nullptr && T > 0) return WINDQ_EINVAL;
    const size_t eb = dY->dtype == WINDQ_F32 ? 4 : 2;
    if (!sizes_fit(T, Q.P.rows, Q.P.cols, Q.A.n, Q.A.max_rank)) return WINDQ_ESHAPE;
    if (dX != nullptr) {
        if (ld_dx < Q.P.cols || ld_dx > (int64_t)1 << 31) return WINDQ_ESHAPE;
        if (!aligned(dX, eb)) return WINDQ_EINVAL;
    }
    const GradWs at = grad_ws(dY->dtype, T, Q.P.rows, Q.P.cols, Q.A.n, Q.A.max_rank);
    if (ws == nullptr || ws_bytes < at.total) return WINDQ_EWORKSPACE;
    if (!aligned(ws, 256)) return WINDQ_EINVAL;
    Q.T = T;
    Q.dX = dX;
    Q.ldx = ld_dx;
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* w = static_cast<char*>(ws);
    return dY->dtype == WINDQ_F32 ? grad_all<float>(Q, dY, X, h, dA, dB, w, at, st) : grad_all<uint16_t>(Q, dY, X, h, dA, dB, w, at, st);
}

