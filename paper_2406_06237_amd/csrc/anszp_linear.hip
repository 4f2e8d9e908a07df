// Matrix product with its epilogue, for gfx950: rows of activations times a layer's weights [cols][k],
//   y[r, c] = act(s_x[r] * s_w[c] * sum_k x[r, k] * w[c, k] + bias[c]) * mul[r, c] + residual[r, c]
// with x and w in bf16 (weights as anszp_decode leaves them), or x in 8 bits with a scale a row and w as symbols, w - z for them
// (Sec. II-B).  bf16 products are exact in the fp32 sums of the matrix instructions, 8-bit ones are summed exactly in 32-bit
// integers.  The matrix instructions take signed bytes, so symbols go in as q - 128 (the top bit flipped) and
//   sum_k x (q - z) = sum_k x (q - 128) + (128 - z) sum_k x,
// the second sum from the same instructions with ones in the weights' place; it is left out where z = 128.
// In the instructions' terms the weights are the rows and the activations the columns of the product, so that a lane ends up
// with four consecutive output channels of one row of activations.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "anszp_cus.h"
#include "anszp_linear_plan.h"
#include "anszp_numbers.h"

namespace {

struct LinearParams {
    const uint8_t* x;
    const uint8_t* w;
    const float* x_scales;
    const float* channel_scales;
    const float* bias;
    const void* mul;
    const void* residual;
    void* out;
    uint64_t x_stride, w_stride;        // bytes between rows
    uint64_t mul_stride, residual_stride, out_stride;   // elements
    uint64_t rows, cols;
    uint32_t k_bytes, activation, out_dtype;
    int32_t offset;                     // 128 - zero_point
    float scale;
    // k in shares: sums of 32 bits, [share][rows][cols up to a multiple of 8], that linear_join_kernel adds up; NULL: none
    uint32_t* parts;
    uint32_t shares, share_steps;       // whole steps of 128 bytes a share has; the last one has what is left of k, too
    uint64_t parts_stride;              // columns of a row
};

// erf to 1.5e-7, which binary32 next to one cannot tell much better (Abramowitz and Stegun, 7.1.26): a third of erff's instructions, and the
// epilogue of large products runs with the matrix units idle.
__device__ __forceinline__ float erf_of(float v) {
    const float x = fabsf(v), t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.0f));
    const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    return copysignf(fmaf(-poly, __builtin_amdgcn_exp2f(x * x * -1.4426950408889634f), 1.0f), v);
}

__device__ __forceinline__ float activated(float v, uint32_t activation) {
    switch (activation) {
        case ANSZP_FN_RELU: return v < 0.0f ? 0.0f : v;
        case ANSZP_FN_GELU: return 0.5f * v * (1.0f + erf_of(v * 0.70710678118654752f));
        case ANSZP_FN_SILU: return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.4426950408889634f));
        default: return v;
    }
}

// N = 4 or 8 consecutive elements of the output's type as they lie in memory, zeros behind the end of a row.  (Whole vectors are set and read in both
// types' ways: where one word or another is, the compiler joins the ways by a place to be worked out, and the words lie in memory.)
template <uint32_t N>
struct Some {
    words4 lo, hi;                                          // bf16: lo alone
    __device__ __forceinline__ void load(const void* base, uint32_t dtype, uint64_t at, uint32_t there) {
        words4 a = {0u, 0u, 0u, 0u}, b = {0u, 0u, 0u, 0u};
        if (dtype == ANSZP_OUT_BF16) {
            const uint16_t* p = static_cast<const uint16_t*>(base) + at;
            if (there >= N) {
                if constexpr (N == 8u) {
                    a = *reinterpret_cast<const words4_any*>(p);
                } else {
                    const words2 t = *reinterpret_cast<const words2_any*>(p);
                    a = words4{t[0], t[1], 0u, 0u};
                }
            } else {
#pragma unroll
                for (uint32_t i = 0; i < N; ++i)
                    if (i < there) a[i / 2u] |= uint32_t(p[i]) << (16u * (i & 1u));
            }
        } else {
            const uint32_t* p = static_cast<const uint32_t*>(base) + at;
            if (there >= N) {
                a = *reinterpret_cast<const words4_any*>(p);
                if constexpr (N == 8u) b = *reinterpret_cast<const words4_any*>(p + 4);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < N; ++i)
                    if (i < there) (i < 4u ? a : b)[i & 3u] = p[i];
            }
        }
        lo = a;
        hi = b;
    }
    __device__ __forceinline__ float at(uint32_t dtype, uint32_t i) const {
        const words4 a = lo, b = hi;
        const uint32_t two = a[i / 2u], one = i < 4u ? a[i & 3u] : b[i & 3u];
        return dtype == ANSZP_OUT_BF16 ? i & 1u ? bf16_high(two) : bf16_low(two) : __builtin_bit_cast(float, one);
    }
};

// The epilogue of N consecutive channels: what belongs to the channels, what belongs to a row of them, and a row's sums to the output.  A row's
// operands are asked for apart from their use, so that those of several rows are under way together (out may be one of them, which
// keeps the compiler from moving a load before a store).
template <uint32_t N>
struct Channels {
    Some<N> scale, bias;
    uint64_t col;
    uint32_t there;
    __device__ __forceinline__ void load(const LinearParams& p, uint64_t from) {
        col = from;
        there = col >= p.cols ? 0u : p.cols - col >= N ? N : uint32_t(p.cols - col);
        if (p.channel_scales) scale.load(p.channel_scales, ANSZP_OUT_F32, col, there);
        if (p.bias) bias.load(p.bias, ANSZP_OUT_F32, col, there);
    }
};
// The operands of a row, in the output's type: one that is known here (eight elements of it), or else p.out_dtype.
constexpr uint32_t kAnyType = ~0u;
template <uint32_t N, uint32_t DTYPE>
struct Operand : Eight<DTYPE> {
    static_assert(N == 8u, "");
    __device__ __forceinline__ float at(uint32_t, uint32_t i) const { return (*this)[i]; }
};
template <uint32_t N>
struct Operand<N, kAnyType> : Some<N> {};
template <uint32_t N, uint32_t DTYPE = kAnyType>
struct RowOperands {
    Operand<N, DTYPE> mul, residual;
    float by;
    __device__ __forceinline__ void load(const LinearParams& p, const Channels<N>& c, uint64_t row) {
        if (row >= p.rows || c.there == 0u) return;
        by = p.x_scales ? p.scale * p.x_scales[row] : p.scale;
        if (p.mul) mul.load(p.mul, p.out_dtype, row * p.mul_stride + c.col, c.there);
        if (p.residual) residual.load(p.residual, p.out_dtype, row * p.residual_stride + c.col, c.there);
    }
};
template <uint32_t N, uint32_t DTYPE>
__device__ __forceinline__ void finish(const LinearParams& p, const Channels<N>& c, const RowOperands<N, DTYPE>& o, uint64_t row, const float (&sum)[N]) {
    const uint32_t dtype = DTYPE == kAnyType ? p.out_dtype : DTYPE;
    if (row >= p.rows || c.there == 0u) return;
    float v[N];
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) v[i] = sum[i] * o.by;
    if (p.channel_scales) {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) v[i] *= c.scale.at(ANSZP_OUT_F32, i);
    }
    if (p.bias) {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) v[i] += c.bias.at(ANSZP_OUT_F32, i);
    }
    if (p.activation) {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) v[i] = activated(v[i], p.activation);
    }
    if (p.mul) {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) v[i] *= o.mul.at(dtype, i);
    }
    if (p.residual) {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) v[i] += o.residual.at(dtype, i);
    }
    const uint64_t to = row * p.out_stride + c.col;
    if (dtype == ANSZP_OUT_BF16) {
        uint16_t* out = static_cast<uint16_t*>(p.out) + to;
        if (c.there >= N) {
            if constexpr (N == 8u)
                *reinterpret_cast<words4_any*>(out) = words4{to_bf16_pair(v[0], v[1]), to_bf16_pair(v[2], v[3]), to_bf16_pair(v[4], v[5]), to_bf16_pair(v[6], v[7])};
            else
                *reinterpret_cast<words2_any*>(out) = words2{to_bf16_pair(v[0], v[1]), to_bf16_pair(v[2], v[3])};
        } else {
#pragma unroll
            for (uint32_t i = 0; i < N; ++i)
                if (i < c.there) out[i] = to_bf16(v[i]);
        }
    } else {
        float* out = static_cast<float*>(p.out) + to;
        if (c.there >= N) {
#pragma unroll
            for (uint32_t i = 0; i < N / 4u; ++i)
                reinterpret_cast<words4_any*>(out)[i] = __builtin_bit_cast(words4, floatx4{v[4u * i], v[4u * i + 1u], v[4u * i + 2u], v[4u * i + 3u]});
        } else {
#pragma unroll
            for (uint32_t i = 0; i < N; ++i)
                if (i < c.there) out[i] = v[i];
        }
    }
}
template <uint32_t N>
__device__ __forceinline__ void finish(const LinearParams& p, uint64_t row, uint64_t col, const float (&sum)[N]) {
    Channels<N> c;
    RowOperands<N> o;
    c.load(p, col);
    o.load(p, c, row);
    finish<N, kAnyType>(p, c, o, row, sum);
}

// 16 bytes of a row from byte `at` on, zeros behind its end.
__device__ __forceinline__ words4 piece_of(const uint8_t* row, uint32_t at, uint32_t row_bytes) {
    if (at + 16u <= row_bytes) return *reinterpret_cast<const words4_any*>(row + at);
    words4 w = {0u, 0u, 0u, 0u};
    for (uint32_t i = 0; i < 16u; ++i)
        if (at + i < row_bytes) w[i >> 2] |= uint32_t(row[at + i]) << (8u * (i & 3u));
    return w;
}

// The same of a row of at least 16 bytes, without a loop: the row's last 16 bytes, moved down by what they start before `at`.
__device__ __forceinline__ words4 piece_of_long(const uint8_t* row, uint32_t at, uint32_t row_bytes) {
    const uint32_t first = at < row_bytes - 16u ? at : row_bytes - 16u, over = at - first;
    words4 w = *reinterpret_cast<const words4_any*>(row + first);
    if (over & 8u) w = words4{w[2], w[3], 0u, 0u};
    if (over & 4u) w = words4{w[1], w[2], w[3], 0u};
    const uint32_t bits = 8u * (over & 3u);
    w = words4{__builtin_amdgcn_alignbit(w[1], w[0], bits), __builtin_amdgcn_alignbit(w[2], w[1], bits), __builtin_amdgcn_alignbit(w[3], w[2], bits), w[3] >> bits};
    return over < 16u ? w : words4{0u, 0u, 0u, 0u};
}

// BYTES: 8-bit operands.  One step over 64 bytes of k.
template <bool BYTES>
struct Sums {
    typedef floatx4 type;
    static __device__ __forceinline__ floatx4 step(words4 w, words4 x, floatx4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), c, 0, 0, 0);
    }
};
template <>
struct Sums<true> {
    typedef intx4 type;
    static __device__ __forceinline__ intx4 step(words4 w, words4 x, intx4 c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(intx4, w), __builtin_bit_cast(intx4, x), c, 0, 0, 0);
    }
};

// Any sizes, strides and alignments: 64 channels x 64 rows a workgroup, four wavefronts with 32 x 32 each, 128 bytes of k at a
// time through LDS.  A row of a tile is 8 pieces of 16 bytes; piece j of row r lies in place j ^ (r & 7), so that the 16 lanes that
// read one piece of 16 rows each meet no bank more than twice.  It is for rows of less than 16 bytes and for strides that the others do not take, where
// the output bounds it: 4096 x 4096 x 7 in bf16 28 us.
template <bool BYTES>
__global__ __launch_bounds__(256) void linear_any_kernel(LinearParams p, uint32_t tiles_c) {
    __shared__ words4 tile[2][64][8];                               // weights, activations
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint64_t c0 = uint64_t(blockIdx.x % tiles_c) * 64u, r0 = uint64_t(blockIdx.x / tiles_c) * 64u;
    typename Sums<BYTES>::type acc[2][2] = {}, ones[2] = {};
    const words4 all_one = {0x01010101u, 0x01010101u, 0x01010101u, 0x01010101u};
    for (uint32_t k0 = 0; k0 < p.k_bytes; k0 += 128u) {
        for (uint32_t i = 0; i < 2u; ++i) {
            const uint32_t n = i * 256u + threadIdx.x, row = n >> 3, j = n & 7u;
            const uint32_t at = k0 + j * 16u;
            words4 w = {0u, 0u, 0u, 0u}, x = {0u, 0u, 0u, 0u};
            if (c0 + row < p.cols && at < p.k_bytes) w = piece_of(p.w + (c0 + row) * p.w_stride, at, p.k_bytes);
            if (r0 + row < p.rows && at < p.k_bytes) x = piece_of(p.x + (r0 + row) * p.x_stride, at, p.k_bytes);
            if constexpr (BYTES)
                for (uint32_t e = 0; e < 4u; ++e) w[e] ^= 0x80808080u;
            tile[0][row][j ^ (row & 7u)] = w;
            tile[1][row][j ^ (row & 7u)] = x;
        }
        __syncthreads();
        for (uint32_t kk = 0; kk < 2u; ++kk) {
            words4 w[2], x[2];
            for (uint32_t i = 0; i < 2u; ++i) {
                const uint32_t at = (lane & 15u) + 16u * i, j = (kk * 4u + (lane >> 4)) ^ (at & 7u);
                w[i] = tile[0][(wave & 1u) * 32u + at][j];
                x[i] = tile[1][(wave >> 1) * 32u + at][j];
            }
            for (uint32_t b = 0; b < 2u; ++b) {
                for (uint32_t a = 0; a < 2u; ++a) acc[a][b] = Sums<BYTES>::step(w[a], x[b], acc[a][b]);
                if constexpr (BYTES) ones[b] = Sums<BYTES>::step(all_one, x[b], ones[b]);
            }
        }
        __syncthreads();
    }
    for (uint32_t a = 0; a < 2u; ++a)
        for (uint32_t b = 0; b < 2u; ++b) {
            float sum[4];
            for (uint32_t i = 0; i < 4u; ++i) {
                if constexpr (BYTES) sum[i] = float(acc[a][b][i] + p.offset * ones[b][i]);
                else sum[i] = acc[a][b][i];
            }
            finish<4u>(p, r0 + (wave >> 1) * 32u + b * 16u + (lane & 15u), c0 + (wave & 1u) * 32u + a * 16u + (lane >> 4) * 4u, sum);
        }
}

// Few rows: the weights are read once, straight into the matrix instructions' registers, and memory is what bounds it.  A workgroup has
// 16 * CH channels and all rows (16 * TOK at most); its wavefronts share k, 256 bytes of a row at a time each, and their sums meet in LDS.
// Lane (c, g), c = lane % 16, g = lane / 16, feeds bytes [64 u + 16 g, 64 u + 16 g + 16) of weight row c and of activation row c.
// Rows of either that do not exist are the last one again; their sums are not stored.  16 x 4096 x 11008 in bf16 takes 22 us, 4.1 TB/s of weights (a
// large copy reaches 4.8), 1 x 11008 x 4096 of bytes 10.5 to 12, 3.8 to 4.3; more rows take more weights' and rows' pieces a CU, not more memory.
template <bool BYTES, uint32_t TOK, uint32_t CH, uint32_t WAVES, uint32_t PIECES>
__global__ __launch_bounds__(WAVES * 64u) void linear_few_kernel(LinearParams p) {
    constexpr uint32_t kPieces = PIECES, kChunk = 64u * kPieces;
    typedef typename Sums<BYTES>::type sums;
    __shared__ sums joined[WAVES][(CH + (BYTES ? 1u : 0u)) * TOK][64];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, c = lane & 15u, g = lane >> 4;
    const uint64_t c0 = uint64_t(blockIdx.x) * (16u * CH), r0 = uint64_t(blockIdx.y) * (16u * TOK);
    const uint8_t *w_row[CH], *x_row[TOK];
#pragma unroll
    for (uint32_t a = 0; a < CH; ++a) w_row[a] = p.w + least(c0 + 16u * a + c, p.cols - 1u) * p.w_stride;
#pragma unroll
    for (uint32_t b = 0; b < TOK; ++b) x_row[b] = p.x + least(r0 + 16u * b + c, p.rows - 1u) * p.x_stride;
    const words4 all_one = {0x01010101u, 0x01010101u, 0x01010101u, 0x01010101u};
    sums acc[CH][TOK] = {}, ones[TOK] = {};
    words4 w[2][CH][kPieces], x[2][TOK][kPieces];
    const auto load = [&](uint32_t slot, uint32_t k0) __attribute__((always_inline)) {
        if (k0 + kChunk <= p.k_bytes) {
#pragma unroll
            for (uint32_t u = 0; u < kPieces; ++u) {
#pragma unroll
                for (uint32_t a = 0; a < CH; ++a) w[slot][a][u] = *reinterpret_cast<const words4_any*>(w_row[a] + k0 + 64u * u + 16u * g);
#pragma unroll
                for (uint32_t b = 0; b < TOK; ++b) x[slot][b][u] = *reinterpret_cast<const words4_any*>(x_row[b] + k0 + 64u * u + 16u * g);
            }
        } else {
#pragma unroll
            for (uint32_t u = 0; u < kPieces; ++u) {
                const uint32_t at = k0 + 64u * u + 16u * g;
#pragma unroll
                for (uint32_t a = 0; a < CH; ++a) w[slot][a][u] = piece_of_long(w_row[a], at, p.k_bytes);
#pragma unroll
                for (uint32_t b = 0; b < TOK; ++b) x[slot][b][u] = piece_of_long(x_row[b], at, p.k_bytes);
            }
        }
    };
    const auto multiply = [&](uint32_t slot) __attribute__((always_inline)) {
#pragma unroll
        for (uint32_t u = 0; u < kPieces; ++u) {
            if constexpr (BYTES)
#pragma unroll
                for (uint32_t a = 0; a < CH; ++a)
#pragma unroll
                    for (uint32_t e = 0; e < 4u; ++e) w[slot][a][u][e] ^= 0x80808080u;
#pragma unroll
            for (uint32_t b = 0; b < TOK; ++b) {
#pragma unroll
                for (uint32_t a = 0; a < CH; ++a) acc[a][b] = Sums<BYTES>::step(w[slot][a][u], x[slot][b][u], acc[a][b]);
                if constexpr (BYTES) ones[b] = Sums<BYTES>::step(all_one, x[slot][b][u], ones[b]);
            }
        }
    };
    uint32_t k0 = wave * kChunk;
    if (k0 < p.k_bytes) load(0u, k0);
    while (k0 < p.k_bytes) {                              // (one piece of k on its way while the other is multiplied)
        k0 += WAVES * kChunk;
        if (k0 < p.k_bytes) load(1u, k0);
        multiply(0u);
        if (k0 >= p.k_bytes) break;
        k0 += WAVES * kChunk;
        if (k0 < p.k_bytes) load(0u, k0);
        multiply(1u);
    }
#pragma unroll
    for (uint32_t b = 0; b < TOK; ++b) {
#pragma unroll
        for (uint32_t a = 0; a < CH; ++a) joined[wave][a * TOK + b][lane] = acc[a][b];
        if constexpr (BYTES) joined[wave][CH * TOK + b][lane] = ones[b];
    }
    __syncthreads();
    for (uint32_t tile = wave; tile < CH * TOK; tile += WAVES) {
        const uint32_t a = tile / TOK, b = tile % TOK;
        sums all = joined[0][tile][lane];
        for (uint32_t v = 1; v < WAVES; ++v) all += joined[v][tile][lane];
        float sum[4];
        if constexpr (BYTES) {
            sums one = joined[0][CH * TOK + b][lane];
            for (uint32_t v = 1; v < WAVES; ++v) one += joined[v][CH * TOK + b][lane];
#pragma unroll
            for (uint32_t i = 0; i < 4u; ++i) sum[i] = float(all[i] + p.offset * one[i]);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 4u; ++i) sum[i] = all[i];
        }
        finish<4u>(p, r0 + b * 16u + c, c0 + a * 16u + g * 4u, sum);
    }
}

template <bool BYTES, uint32_t TOK, uint32_t CH, uint32_t PIECES>
bool launch_few(const LinearParams& p, hipStream_t s) {
    constexpr uint32_t kWaves = 8u;
    const uint64_t groups_c = (p.cols + 16u * CH - 1u) / (16u * CH), groups_t = (p.rows + 16u * TOK - 1u) / (16u * TOK);
    if (groups_c * (kWaves * 64u) >= 1ull << 32 || groups_t > 65535u) return false;
    hipLaunchKernelGGL((linear_few_kernel<BYTES, TOK, CH, kWaves, PIECES>), dim3(static_cast<uint32_t>(groups_c), static_cast<uint32_t>(groups_t)), dim3(kWaves * 64u), 0, s, p);
    return true;
}

// Many rows: TOK activations' rows x CH channels a workgroup of WT x WC wavefronts, v_mfma_*_32x32, k in steps of 128 bytes through two
// buffers in LDS.  A row of a buffer is 8 pieces of 16 bytes; piece j of row r lies in place j ^ (r / 2 % 8), so that 16 lanes that read one
// piece of neighbouring rows meet all 64 banks.
// DIRECT: rows begin at multiples of 16 bytes, and steps go from memory to LDS without passing through registers; a wavefront's load fills 8
// rows end to end, each lane asking for the piece that belongs where its 16 bytes land.  Otherwise, and for what is left of k behind the last
// whole step, pieces are loaded to registers, with zeros behind the end of a row.  256 x 256 tiles have too few for that (42 spill in 8 bits, 18 in bf16):
// 8192 x 4096 x 4096 takes 252 us in bf16 and 148 in 8 bits, with k of 4095 289 and 225.
typedef __attribute__((ext_vector_type(16))) float floatx16;
typedef __attribute__((ext_vector_type(16))) int32_t intx16;
template <bool BYTES>
struct Sums32 {
    typedef floatx16 type;
    static __device__ __forceinline__ floatx16 step(words4 w, words4 x, floatx16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), c, 0, 0, 0);
    }
};
template <>
struct Sums32<true> {
    typedef intx16 type;
    static __device__ __forceinline__ intx16 step(words4 w, words4 x, intx16 c) {
        return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(intx4, w), __builtin_bit_cast(intx4, x), c, 0, 0, 0);
    }
};

typedef __attribute__((address_space(1))) const void global_void;
typedef __attribute__((address_space(3))) void lds_void;

// Workgroups go to the chip's eight dies in turn, and each die has an L2 of its own: those of one die get neighbouring tiles, columns of
// kPanel tiles one behind the other, so that the 32 tiles a die works on at a time share 8 + 4 blocks of rows.
constexpr uint32_t kDies = 8u, kPanel = 8u;
__device__ __forceinline__ void place_tile(uint32_t block, uint32_t tiles_t, uint32_t tiles_c, uint32_t& tile_t, uint32_t& tile_c) {
    const uint32_t n = tiles_t * tiles_c, die = block % kDies;
    const uint32_t at = die * (n / kDies) + (die < n % kDies ? die : n % kDies) + block / kDies;
    const uint32_t panel = at / (kPanel * tiles_c), in = at - panel * kPanel * tiles_c;
    const uint32_t left = tiles_t - panel * kPanel, high = left < kPanel ? left : kPanel;
    tile_c = in / high;
    tile_t = panel * kPanel + in % high;
}

template <bool BYTES, bool DIRECT, uint32_t TOK, uint32_t CH, uint32_t WT, uint32_t WC, uint32_t STAGES>
__global__ __launch_bounds__(WT * WC * 64u) void linear_tile_kernel(LinearParams p, uint32_t tiles_c, uint32_t tiles_t) {
    constexpr uint32_t kThreads = WT * WC * 64u, kRows = TOK + CH, kFT = TOK / WT / 32u, kFC = CH / WC / 32u;
    constexpr uint32_t kStepBytes = 128u, kLoads = kRows * 8u / kThreads, kHalf = kLoads / 2u;      // pieces a thread brings per step
    static_assert(kRows * 8u % kThreads == 0u && TOK * 8u % kThreads == 0u, "a load is of one operand");
    __shared__ words4 buffer[STAGES][kRows][8];                            // activations, then weights
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wt = wave / WC, wc = wave % WC;
    uint32_t tile_t, tile_c;
    place_tile(blockIdx.x, tiles_t, tiles_c, tile_t, tile_c);
    const uint64_t t0 = uint64_t(tile_t) * TOK, c0 = uint64_t(tile_c) * CH;

    // Where this thread's pieces come from: bytes behind the tile's first row of activations or weights (rows that do not exist are the last one
    // again), for a step with what of k lies before it.
    const uint32_t all_whole = p.k_bytes / kStepBytes, before = blockIdx.y * p.share_steps;      // steps of the shares before this one
    const uint8_t *const x_tile = p.x + t0 * p.x_stride + before * kStepBytes, *const w_tile = p.w + c0 * p.w_stride + before * kStepBytes;
    const uint32_t x_last = uint32_t(least(p.rows - t0, TOK) - 1u), w_last = uint32_t(least(p.cols - c0, CH) - 1u);
    const uint32_t piece = 16u * ((threadIdx.x & 7u) ^ ((threadIdx.x >> 4) & 7u));
    uint32_t from[kLoads];
#pragma unroll
    for (uint32_t i = 0; i < kLoads; ++i) {
        const uint32_t row = (i * kThreads + threadIdx.x) >> 3;
        from[i] = i * kThreads < TOK * 8u ? min(row, x_last) * uint32_t(p.x_stride) : min(row - TOK, w_last) * uint32_t(p.w_stride);
    }
    const auto operand = [&](uint32_t i) __attribute__((always_inline)) { return i * kThreads < TOK * 8u ? x_tile : w_tile; };
    // Step 0 is what is left of k behind the whole steps, if anything.
    const uint32_t whole = min(p.share_steps, all_whole - before), rest = blockIdx.y + 1u == p.shares && p.k_bytes % kStepBytes ? 1u : 0u, steps = whole + rest;
    const uint32_t row_end = p.k_bytes - before * kStepBytes;
    words4 held[kLoads];
    const auto load = [&](uint32_t s) __attribute__((always_inline)) {
        if (s >= steps) return;
        if (s < rest) {
#pragma unroll
            for (uint32_t i = 0; i < kLoads; ++i) held[i] = piece_of_long(operand(i) + from[i], whole * kStepBytes + piece, row_end);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < kLoads; ++i) held[i] = *reinterpret_cast<const words4_any*>(operand(i) + (s - rest) * kStepBytes + (from[i] + piece));
        }
    };
    const auto put = [&](uint32_t s) __attribute__((always_inline)) {
        if (s >= steps) return;
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i) buffer[s & (STAGES - 1u)][(i * kThreads + threadIdx.x) >> 3][threadIdx.x & 7u] = held[i];
    };
    const auto bring = [&](uint32_t s, uint32_t begin, uint32_t end) __attribute__((always_inline)) {      // loads of a whole step
#pragma unroll
        for (uint32_t i = begin; i < end; ++i)
            __builtin_amdgcn_global_load_lds((global_void*)(operand(i) + (s - rest) * kStepBytes + (from[i] + piece)),
                                             (lds_void*)(&buffer[s & (STAGES - 1u)][(i * kThreads + wave * 64u) >> 3][0]), 16, 0, 0);
    };
    // The step behind is there for all wavefronts, and what they read before has been read.  No barrier waits by itself for loads that go to LDS.
    const auto arrived = [&]() __attribute__((always_inline)) {
        if constexpr (DIRECT) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    typename Sums32<BYTES>::type acc[kFC][kFT] = {};
    int32_t x_sums[kFT] = {};
    words4 x[2][kFT], w[2][kFC];
    const uint32_t r = lane & 31u;
    const auto fetch = [&](uint32_t slot, uint32_t s, uint32_t kk) __attribute__((always_inline)) {
        const uint32_t j = (kk * 2u + (lane >> 5)) ^ ((r >> 1) & 7u);
#pragma unroll
        for (uint32_t f = 0; f < kFC; ++f) w[slot][f] = buffer[s & (STAGES - 1u)][TOK + wc * (CH / WC) + f * 32u + r][j];
#pragma unroll
        for (uint32_t f = 0; f < kFT; ++f) x[slot][f] = buffer[s & (STAGES - 1u)][wt * (TOK / WT) + f * 32u + r][j];
    };
    // A quarter of a step; between(a) comes behind the instructions of the a-th rows of channels.
    const auto multiply = [&](uint32_t slot, auto between) __attribute__((always_inline)) {
#pragma unroll
        for (uint32_t a = 0; a < kFC; ++a) {
            if constexpr (BYTES) {
#pragma unroll
                for (uint32_t e = 0; e < 4u; ++e) w[slot][a][e] ^= 0x80808080u;
            }
#pragma unroll
            for (uint32_t b = 0; b < kFT; ++b) {
                acc[a][b] = Sums32<BYTES>::step(w[slot][a], x[slot][b], acc[a][b]);
                if constexpr (BYTES) {                                       // a word of each piece behind each row of channels
#pragma unroll
                    for (uint32_t e = 0; e < 4u; ++e)
                        if (e * kFC / 4u == a) x_sums[b] = __builtin_amdgcn_sdot4(int32_t(x[slot][b][e]), 0x01010101, x_sums[b], false);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            between(a);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // The operands of the next quarter of a step are on their way to registers while this one's are multiplied.  Before a step's last quarter is
    // multiplied every wavefront has all it needs of the step's buffer: from there on it takes the step after the next.  Its loads are spread
    // over that quarter and the next one (asked for in one go they keep the wavefront from multiplying), which leaves them half a step to arrive.
    constexpr bool kDeep = DIRECT && STAGES > 2u;
    constexpr uint32_t kAhead = STAGES - 1u;
    load(0u);
    put(0u);
    if constexpr (kDeep) {
#pragma unroll
        for (uint32_t i = 1; i < kAhead; ++i)
            if (i < steps) bring(i, 0u, kLoads);
    } else if constexpr (DIRECT) {
        if (1u < steps) bring(1u, 0u, kHalf);
    } else {
        load(1u);
    }
    __syncthreads();
    fetch(0u, 0u, 0u);
    const auto step = [&](uint32_t s, auto more) __attribute__((always_inline)) {
        constexpr bool kMore = decltype(more)::value;                        // two steps are still to come
        multiply(0u, [&](uint32_t a) __attribute__((always_inline)) {
            if (a == 0u) fetch(1u, s, 1u);
            if (DIRECT && (kMore || s + 1u < steps)) bring(s + 1u, kHalf + a * (kLoads - kHalf) / kFC, kHalf + (a + 1u) * (kLoads - kHalf) / kFC);
            if (!DIRECT && a + 1u == kFC) put(s + 1u);
        });
        multiply(1u, [&](uint32_t a) __attribute__((always_inline)) {
            if (a == 0u) fetch(0u, s, 2u);
            if (!DIRECT && a + 1u == kFC) load(s + 2u);
        });
        multiply(0u, [&](uint32_t a) __attribute__((always_inline)) {
            if (a == 0u) fetch(1u, s, 3u);
        });
        arrived();
        if (kMore || s + 1u < steps) fetch(0u, s + 1u, 0u);
        __builtin_amdgcn_sched_barrier(0);
        multiply(1u, [&](uint32_t a) __attribute__((always_inline)) {
            if (DIRECT && kMore) bring(s + 2u, a * kHalf / kFC, (a + 1u) * kHalf / kFC);
        });
    };
    // With more buffers than two a step's loads are under way for kAhead - 1 steps; the buffer they go to is that of the step before this one.
    const auto step_deep = [&](uint32_t s, auto more) __attribute__((always_inline)) {
        constexpr bool kMore = decltype(more)::value;                        // kAhead steps are still to come
        const auto third = [&](uint32_t n, uint32_t a) __attribute__((always_inline)) {
            if (kMore && a == 0u) bring(s + kAhead, n * kLoads / 3u, (n + 1u) * kLoads / 3u);
        };
        multiply(0u, [&](uint32_t a) __attribute__((always_inline)) {
            if (a == 0u) fetch(1u, s, 1u);
            third(0u, a);
        });
        multiply(1u, [&](uint32_t a) __attribute__((always_inline)) {
            if (a == 0u) fetch(0u, s, 2u);
            third(1u, a);
        });
        multiply(0u, [&](uint32_t a) __attribute__((always_inline)) {
            if (a == 0u) fetch(1u, s, 3u);
            third(2u, a);
        });
        // (A barrier of the language's own would wait for all loads that go to LDS.)
        if constexpr (kMore) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((kAhead - 1u) * kLoads) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (kMore || s + 1u < steps) fetch(0u, s + 1u, 0u);
        __builtin_amdgcn_sched_barrier(0);
        multiply(1u, [](uint32_t) {});
    };
    uint32_t s = 0u;
    if constexpr (kDeep) {
        for (; s + kAhead < steps; ++s) step_deep(s, std::true_type{});
        for (; s < steps; ++s) step_deep(s, std::false_type{});
    } else {
        for (; s + 2u < steps; ++s) step(s, std::true_type{});
        for (; s < steps; ++s) step(s, std::false_type{});
    }

    // To the output through LDS, 32 rows of a wavefront's channels at a time, so that a row's channels are stored end to end (and mul and
    // residual read so); four channels of row r lie in place (channel / 4) ^ (r & 7).
    constexpr uint32_t kWidth = CH / WC, kLanes = kWidth / 8u;               // channels of a wavefront; lanes that have a row of them
    static_assert(WT * WC * 32u * kWidth * 4u <= sizeof(buffer) && 64u % kLanes == 0u, "the epilogue's part of LDS");
    floatx4(*part)[kWidth / 4u] = reinterpret_cast<floatx4(*)[kWidth / 4u]>(reinterpret_cast<uint8_t*>(buffer) + wave * (32u * kWidth * 4u));
    const uint32_t own = lane % kLanes;
    const uint64_t first = t0 + wt * (TOK / WT);
    Channels<8u> channels;
    channels.load(p, c0 + wc * kWidth + own * 8u);
    __syncthreads();
#pragma unroll
    for (uint32_t b = 0; b < kFT; ++b) {
        int32_t more = 0;
        if constexpr (BYTES) more = p.offset * (x_sums[b] + __shfl_xor(x_sums[b], 32));
#pragma unroll
        for (uint32_t a = 0; a < kFC; ++a)
#pragma unroll
            for (uint32_t i = 0; i < 4u; ++i) {
                floatx4 four;
#pragma unroll
                for (uint32_t e = 0; e < 4u; ++e) {
                    if constexpr (BYTES) {
                        const int32_t sum = acc[a][b][4u * i + e] + more;
                        four[e] = p.parts ? __builtin_bit_cast(float, sum) : float(sum);
                    } else {
                        four[e] = acc[a][b][4u * i + e];
                    }
                }
                part[r][(a * 8u + 2u * i + (lane >> 5)) ^ (r & 7u)] = four;
            }
        __builtin_amdgcn_wave_barrier();
        constexpr uint32_t kRowsAtOnce = 64u / kLanes, kTurns = 32u / kRowsAtOnce;
        const auto row_of = [&](uint32_t turn) __attribute__((always_inline)) { return turn * kRowsAtOnce + lane / kLanes; };
        const auto store = [&](uint32_t turn, const RowOperands<8u>& operands) __attribute__((always_inline)) {
            const uint32_t n = row_of(turn);
            const floatx4 lo = part[n][(2u * own) ^ (n & 7u)], hi = part[n][(2u * own + 1u) ^ (n & 7u)];
            const uint64_t row = first + b * 32u + n;
            if (p.parts) {
                if (row < p.rows && channels.there) {
                    floatx4* const to = reinterpret_cast<floatx4*>(p.parts + (blockIdx.y * p.rows + row) * p.parts_stride + channels.col);
                    to[0] = lo;
                    to[1] = hi;
                }
            } else {
                const float sum[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                finish<8u, kAnyType>(p, channels, operands, row, sum);
            }
        };
        static_assert(kTurns % 2u == 0u, "two turns' operands at once");
        if (!p.parts && p.out_dtype == ANSZP_OUT_BF16 && c0 + (wc + 1u) * kWidth <= p.cols) {
            // What 32 rows need of memory is asked for together, under no condition of a lane's own (rows that do not exist are the last one again), before any
            // is finished: 8192 x 11008 x 4096 of bytes with mul took 536 us with two rows under way, 466 with 32; 3001 x 4096 x 4096 with a residual 110 and 103.
            RowOperands<8u, ANSZP_OUT_BF16> operands[kTurns];
            Channels<8u> all = channels;
            all.there = 8u;
            const auto existing = [&](uint32_t turn) __attribute__((always_inline)) { return least(first + b * 32u + row_of(turn), p.rows - 1u); };
            if (p.mul) {
#pragma unroll
                for (uint32_t turn = 0; turn < kTurns; ++turn) operands[turn].mul.load(p.mul, existing(turn) * p.mul_stride + all.col, 8u);
            }
            if (p.residual) {
#pragma unroll
                for (uint32_t turn = 0; turn < kTurns; ++turn) operands[turn].residual.load(p.residual, existing(turn) * p.residual_stride + all.col, 8u);
            }
#pragma unroll
            for (uint32_t turn = 0; turn < kTurns; ++turn) operands[turn].by = p.x_scales ? p.scale * p.x_scales[existing(turn)] : p.scale;
#pragma unroll
            for (uint32_t turn = 0; turn < kTurns; ++turn) {
                const uint32_t n = row_of(turn);
                const floatx4 lo = part[n][(2u * own) ^ (n & 7u)], hi = part[n][(2u * own + 1u) ^ (n & 7u)];
                const float sum[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                finish<8u, ANSZP_OUT_BF16>(p, all, operands[turn], first + b * 32u + n, sum);
            }
            __builtin_amdgcn_wave_barrier();
            continue;
        }
        for (uint32_t turn = 0; turn < kTurns; turn += 2u) {
            RowOperands<8u> one, two;
            if (!p.parts) {
                one.load(p, channels, first + b * 32u + row_of(turn));
                two.load(p, channels, first + b * 32u + row_of(turn + 1u));
            }
            store(turn, one);
            store(turn + 1u, two);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// The shares' sums together, eight channels a thread, and the epilogue.  Partial sums are read once, end to end: 64 x 4096 x 11008 in bf16 takes 27 us with
// eight shares and this, 42 with the best kernel that has none.
template <bool BYTES>
__global__ __launch_bounds__(256) void linear_join_kernel(LinearParams p) {
    const uint64_t n = (uint64_t(blockIdx.x) * 256u + threadIdx.x) * 8u, row = n / p.parts_stride, col = n - row * p.parts_stride;
    if (row >= p.rows) return;
    typedef typename Sums<BYTES>::type sums;
    const sums* from = reinterpret_cast<const sums*>(p.parts + n);
    sums lo = from[0], hi = from[1];
    for (uint32_t s = 1; s < p.shares; ++s) {
        from = reinterpret_cast<const sums*>(p.parts + s * p.rows * p.parts_stride + n);
        lo += from[0];
        hi += from[1];
    }
    const float sum[8] = {float(lo[0]), float(lo[1]), float(lo[2]), float(lo[3]), float(hi[0]), float(hi[1]), float(hi[2]), float(hi[3])};
    finish<8u>(p, row, col, sum);
}

template <bool BYTES, uint32_t TOK, uint32_t CH, uint32_t WT, uint32_t WC, uint32_t STAGES>
bool launch_tile(const LinearParams& p, bool direct, hipStream_t s) {
    const uint64_t tiles_c = (p.cols + CH - 1u) / CH, tiles_t = (p.rows + TOK - 1u) / TOK, joins = (p.rows * p.parts_stride / 8u + 255u) / 256u;
    if (tiles_c * tiles_t * (WT * WC * 64u) >= 1ull << 32 || (p.parts && joins * 256u >= 1ull << 32)) return false;
    const dim3 grid(static_cast<uint32_t>(tiles_c * tiles_t), p.shares), threads(WT * WC * 64u);
    const uint32_t c = static_cast<uint32_t>(tiles_c), t = static_cast<uint32_t>(tiles_t);
    // Four buffers, three steps' loads under way, where all workgroups that have them find place, two a CU: few others fill a workgroup's waits then.  In
    // bf16, us with two buffers and with four: 64 x 4096 x 4096 15.0 and 12.7, 64 x 11008 x 4096 34 and 29.5; with more workgroups (256 x 4096 x 4096
    // in four shares, 1024 of them) 24.1 and 26.9.
    const bool deep = STAGES > 2u && tiles_c * tiles_t * p.shares <= 2u * device_cus();
    if (direct && deep) hipLaunchKernelGGL((linear_tile_kernel<BYTES, true, TOK, CH, WT, WC, STAGES>), grid, threads, 0, s, p, c, t);
    else if (direct) hipLaunchKernelGGL((linear_tile_kernel<BYTES, true, TOK, CH, WT, WC, 2u>), grid, threads, 0, s, p, c, t);
    else hipLaunchKernelGGL((linear_tile_kernel<BYTES, false, TOK, CH, WT, WC, 2u>), grid, threads, 0, s, p, c, t);
    if (p.parts) hipLaunchKernelGGL(linear_join_kernel<BYTES>, dim3(static_cast<uint32_t>(joins)), dim3(256), 0, s, p);
    return true;
}

template <bool BYTES>
bool launch(const LinearParams& p, LinearKernel kernel, hipStream_t s) {
    const bool direct = ((reinterpret_cast<uintptr_t>(p.x) | reinterpret_cast<uintptr_t>(p.w) | p.x_stride | p.w_stride) & 15u) == 0u;
    switch (kernel) {
        case kFew11: return launch_few<BYTES, 1u, 1u, 4u>(p, s);
        case kFew21: return launch_few<BYTES, 2u, 1u, 2u>(p, s);
        case kFew22: return launch_few<BYTES, 2u, 2u, 2u>(p, s);
        case kFew24: return launch_few<BYTES, 2u, 4u, 2u>(p, s);
        case kTile64: return launch_tile<BYTES, 64u, 64u, 2u, 2u, 4u>(p, direct, s);
        case kTile128: return launch_tile<BYTES, 128u, 128u, 2u, 2u, 2u>(p, direct, s);
        case kTile192: return launch_tile<BYTES, 192u, 256u, 2u, 4u, 2u>(p, direct, s);
        case kTile256: return launch_tile<BYTES, 256u, 256u, 4u, 2u, 2u>(p, direct, s);
        default: break;
    }
    const uint64_t tiles_c = (p.cols + 63u) / 64u, tiles_t = (p.rows + 63u) / 64u;
    if (tiles_c * tiles_t * 256u >= 1ull << 32) return false;               // (what is beyond would be left out without an error)
    hipLaunchKernelGGL(linear_any_kernel<BYTES>, dim3(static_cast<uint32_t>(tiles_c * tiles_t)), dim3(256), 0, s, p, static_cast<uint32_t>(tiles_c));
    return true;
}

// The call's parameters but for its shares of k; an error code.
int linear_params(const anszp_linear_args_t& a, LinearParams& p) {
    const bool bytes = a.x_dtype == ANSZP_I8;
    if ((!bytes && a.x_dtype != ANSZP_OUT_BF16) || (a.out_dtype != ANSZP_OUT_F32 && a.out_dtype != ANSZP_OUT_BF16) || a.activation > ANSZP_FN_SILU ||
        a.k == 0 || a.k > (bytes ? 65536u : 1u << 30) || a.rows >= 1ull << 31 || a.cols >= 1ull << 31 || a.zero_point > 255u)
        return ANSZP_E_RANGE;
    if (a.rows > 1 && a.out_stride < a.cols) return ANSZP_E_RANGE;
    const uint32_t size = bytes ? 1u : 2u;
    p = {};
    p.x = static_cast<const uint8_t*>(a.x); p.w = static_cast<const uint8_t*>(a.weight); p.x_scales = a.x_scales; p.channel_scales = a.channel_scales;
    p.bias = a.bias; p.mul = a.mul; p.residual = a.residual; p.out = a.out;
    p.x_stride = a.rows > 1 ? a.x_stride * size : 0u; p.w_stride = a.cols > 1 ? a.weight_stride * size : 0u;      // (the stride of a single row says nothing)
    p.mul_stride = a.mul_stride; p.residual_stride = a.residual_stride; p.out_stride = a.out_stride;
    p.rows = a.rows; p.cols = a.cols; p.k_bytes = a.k * size; p.activation = a.activation; p.out_dtype = a.out_dtype;
    p.offset = 128 - static_cast<int32_t>(a.zero_point); p.scale = a.scale;
    return ANSZP_OK;
}

LinearPlan plan_of(const anszp_linear_args_t& a, const LinearParams& p, bool may_share) {
    return linear_plan(a.x_dtype == ANSZP_I8, p.rows, p.cols, p.k_bytes, p.x_stride, p.w_stride, device_cus(), may_share);
}

}  // namespace

extern "C" uint64_t anszp_linear_workspace_bytes(const anszp_linear_args_t* a) {
    LinearParams p;
    if (!a || linear_params(*a, p) || a->rows == 0 || a->cols == 0) return 0u;
    return plan_of(*a, p, true).workspace;
}

extern "C" int anszp_linear(const anszp_linear_args_t* a, void* hip_stream) {
    if (!a) return ANSZP_E_NULL;
    LinearParams p;
    const int rc = linear_params(*a, p);
    if (rc) return rc;
    if (a->rows == 0 || a->cols == 0) return ANSZP_OK;
    if (!a->x || !a->weight || !a->out) return ANSZP_E_NULL;
    const uint64_t size = a->out_dtype == ANSZP_OUT_BF16 ? 2u : 4u, width = a->cols * size;
    const Rows out = {a->out, a->rows, a->out_stride * size, width};
    if (meet(out, {p.x, p.rows, p.x_stride, p.k_bytes}) || meet(out, {p.w, p.cols, p.w_stride, p.k_bytes}) ||
        meet_elsewhere(out, {a->mul, a->rows, a->mul_stride * size, width}) || meet_elsewhere(out, {a->residual, a->rows, a->residual_stride * size, width}))
        return ANSZP_E_RANGE;
    const LinearPlan plan = plan_of(*a, p, a->workspace != nullptr);
    if (plan.workspace && (a->workspace_bytes < plan.workspace || (reinterpret_cast<uintptr_t>(a->workspace) & 15u))) return ANSZP_E_RANGE;
    p.shares = plan.shares;
    p.share_steps = plan.share_steps;
    p.parts_stride = plan.parts_stride;
    p.parts = plan.shares > 1u ? static_cast<uint32_t*>(a->workspace) : nullptr;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (!(a->x_dtype == ANSZP_I8 ? launch<true>(p, plan.kernel, s) : launch<false>(p, plan.kernel, s))) return ANSZP_E_RANGE;
    return hipGetLastError() == hipSuccess ? ANSZP_OK : ANSZP_E_HIP;
}
