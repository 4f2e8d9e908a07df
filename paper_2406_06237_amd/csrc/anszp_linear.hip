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
};

__device__ __forceinline__ float activated(float v, uint32_t activation) {
    switch (activation) {
        case ANSZP_FN_RELU: return v < 0.0f ? 0.0f : v;
        case ANSZP_FN_GELU: return 0.5f * v * (1.0f + erff(v * 0.70710678118654752f));
        case ANSZP_FN_SILU: return v / (1.0f + expf(-v));
        default: return v;
    }
}

__device__ __forceinline__ void load_four(const void* base, uint32_t dtype, uint64_t at, uint32_t there, float (&v)[4]) {
    if (dtype == ANSZP_OUT_BF16) {
        const uint16_t* p = static_cast<const uint16_t*>(base) + at;
        if (there >= 4u) {
            const words2 w = *reinterpret_cast<const words2_any*>(p);
            v[0] = bf16_low(w[0]); v[1] = bf16_high(w[0]); v[2] = bf16_low(w[1]); v[3] = bf16_high(w[1]);
        } else {
            for (uint32_t i = 0; i < 4u; ++i) v[i] = i < there ? bf16_low(p[i]) : 0.0f;
        }
    } else {
        const float* p = static_cast<const float*>(base) + at;
        if (there >= 4u) {
            const floatx4 w = __builtin_bit_cast(floatx4, *reinterpret_cast<const words4_any*>(p));
            for (uint32_t i = 0; i < 4u; ++i) v[i] = w[i];
        } else {
            for (uint32_t i = 0; i < 4u; ++i) v[i] = i < there ? p[i] : 0.0f;
        }
    }
}

// Four consecutive channels of a row, sums in 32 bits, to the output.
__device__ __forceinline__ void finish_four(const LinearParams& p, uint64_t row, uint64_t col, const float (&sum)[4]) {
    if (row >= p.rows || col >= p.cols) return;
    const uint32_t there = p.cols - col >= 4u ? 4u : uint32_t(p.cols - col);
    const float by = p.x_scales ? p.scale * p.x_scales[row] : p.scale;
    float v[4], t[4];
    for (uint32_t i = 0; i < 4u; ++i) {
        v[i] = sum[i] * by;
        if (p.channel_scales && i < there) v[i] *= p.channel_scales[col + i];
        if (p.bias && i < there) v[i] += p.bias[col + i];
        v[i] = activated(v[i], p.activation);
    }
    if (p.mul) {
        load_four(p.mul, p.out_dtype, row * p.mul_stride + col, there, t);
        for (uint32_t i = 0; i < 4u; ++i) v[i] *= t[i];
    }
    if (p.residual) {
        load_four(p.residual, p.out_dtype, row * p.residual_stride + col, there, t);
        for (uint32_t i = 0; i < 4u; ++i) v[i] += t[i];
    }
    const uint64_t to = row * p.out_stride + col;
    if (p.out_dtype == ANSZP_OUT_BF16) {
        uint16_t* out = static_cast<uint16_t*>(p.out) + to;
        if (there >= 4u) {
            *reinterpret_cast<words2_any*>(out) = words2{to_bf16_pair(v[0], v[1]), to_bf16_pair(v[2], v[3])};
        } else {
            for (uint32_t i = 0; i < 4u; ++i)
                if (i < there) out[i] = to_bf16(v[i]);
        }
    } else {
        float* out = static_cast<float*>(p.out) + to;
        if (there >= 4u) {
            *reinterpret_cast<words4_any*>(out) = __builtin_bit_cast(words4, floatx4{v[0], v[1], v[2], v[3]});
        } else {
            for (uint32_t i = 0; i < 4u; ++i)
                if (i < there) out[i] = v[i];
        }
    }
}

// 16 bytes of a row from byte `at` on, zeros behind its end.
__device__ __forceinline__ words4 piece_of(const uint8_t* row, uint32_t at, uint32_t row_bytes) {
    if (at + 16u <= row_bytes) return *reinterpret_cast<const words4_any*>(row + at);
    words4 w = {0u, 0u, 0u, 0u};
    for (uint32_t i = 0; i < 16u; ++i)
        if (at + i < row_bytes) w[i >> 2] |= uint32_t(row[at + i]) << (8u * (i & 3u));
    return w;
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
// read one piece of 16 rows each meet no bank more than twice.
template <bool BYTES>
__global__ __launch_bounds__(256) void linear_any_kernel(LinearParams p) {
    __shared__ words4 tile[2][64][8];                               // weights, activations
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint64_t c0 = uint64_t(blockIdx.x) * 64u, r0 = uint64_t(blockIdx.y) * 64u;
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
            finish_four(p, r0 + (wave >> 1) * 32u + b * 16u + (lane & 15u), c0 + (wave & 1u) * 32u + a * 16u + (lane >> 4) * 4u, sum);
        }
}

// Few rows: the weights are read once, straight into the matrix instructions' registers, and memory is what bounds it.  A workgroup has
// 16 * CH channels and all rows (16 * TOK at most); its wavefronts share k, 256 bytes of a row at a time each, and their sums meet in LDS.
// Lane (c, g), c = lane % 16, g = lane / 16, feeds bytes [64 u + 16 g, 64 u + 16 g + 16) of weight row c and of activation row c.
// Rows of either that do not exist are the last one again; their sums are not stored.
template <bool BYTES, uint32_t TOK, uint32_t CH, uint32_t WAVES>
__global__ __launch_bounds__(WAVES * 64u) void linear_few_kernel(LinearParams p) {
    constexpr uint32_t kPieces = 4u, kChunk = 64u * kPieces;
    typedef typename Sums<BYTES>::type sums;
    __shared__ sums joined[WAVES][(CH + (BYTES ? 1u : 0u)) * TOK][64];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, c = lane & 15u, g = lane >> 4;
    const uint64_t c0 = uint64_t(blockIdx.x) * (16u * CH), r0 = uint64_t(blockIdx.y) * (16u * TOK);
    const uint8_t *w_row[CH], *x_row[TOK];
    for (uint32_t a = 0; a < CH; ++a) w_row[a] = p.w + least(c0 + 16u * a + c, p.cols - 1u) * p.w_stride;
    for (uint32_t b = 0; b < TOK; ++b) x_row[b] = p.x + least(r0 + 16u * b + c, p.rows - 1u) * p.x_stride;
    const words4 all_one = {0x01010101u, 0x01010101u, 0x01010101u, 0x01010101u};
    sums acc[CH][TOK] = {}, ones[TOK] = {};
    words4 w[2][CH][kPieces], x[2][TOK][kPieces];
    const auto load = [&](uint32_t slot, uint32_t k0) {
        if (k0 + kChunk <= p.k_bytes) {
            for (uint32_t u = 0; u < kPieces; ++u) {
                for (uint32_t a = 0; a < CH; ++a) w[slot][a][u] = *reinterpret_cast<const words4_any*>(w_row[a] + k0 + 64u * u + 16u * g);
                for (uint32_t b = 0; b < TOK; ++b) x[slot][b][u] = *reinterpret_cast<const words4_any*>(x_row[b] + k0 + 64u * u + 16u * g);
            }
        } else {
            for (uint32_t u = 0; u < kPieces; ++u) {
                const uint32_t at = k0 + 64u * u + 16u * g;
                const bool there = at < p.k_bytes;
                for (uint32_t a = 0; a < CH; ++a) w[slot][a][u] = there ? piece_of(w_row[a], at, p.k_bytes) : words4{0u, 0u, 0u, 0u};
                for (uint32_t b = 0; b < TOK; ++b) x[slot][b][u] = there ? piece_of(x_row[b], at, p.k_bytes) : words4{0u, 0u, 0u, 0u};
            }
        }
    };
    const auto multiply = [&](uint32_t slot) {
        for (uint32_t u = 0; u < kPieces; ++u) {
            if constexpr (BYTES)
                for (uint32_t a = 0; a < CH; ++a)
                    for (uint32_t e = 0; e < 4u; ++e) w[slot][a][u][e] ^= 0x80808080u;
            for (uint32_t b = 0; b < TOK; ++b) {
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
    for (uint32_t b = 0; b < TOK; ++b) {
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
            for (uint32_t i = 0; i < 4u; ++i) sum[i] = float(all[i] + p.offset * one[i]);
        } else {
            for (uint32_t i = 0; i < 4u; ++i) sum[i] = all[i];
        }
        finish_four(p, r0 + b * 16u + c, c0 + a * 16u + g * 4u, sum);
    }
}

template <bool BYTES, uint32_t TOK, uint32_t CH, uint32_t WAVES>
void launch_few(const LinearParams& p, hipStream_t s) {
    const dim3 grid(static_cast<uint32_t>((p.cols + 16u * CH - 1u) / (16u * CH)), static_cast<uint32_t>((p.rows + 16u * TOK - 1u) / (16u * TOK)));
    hipLaunchKernelGGL((linear_few_kernel<BYTES, TOK, CH, WAVES>), grid, dim3(WAVES * 64u), 0, s, p);
}

template <bool BYTES>
bool take_few(const LinearParams& p, hipStream_t s) {
    if (p.rows <= 16u) launch_few<BYTES, 1u, 1u, 8u>(p, s);
    else if (p.rows <= 32u) launch_few<BYTES, 2u, 1u, 8u>(p, s);
    else if (p.rows <= 64u) launch_few<BYTES, 4u, 1u, 8u>(p, s);
    else return false;
    return true;
}

}  // namespace

extern "C" int anszp_linear(const anszp_linear_args_t* a, void* hip_stream) {
    if (!a) return ANSZP_E_NULL;
    const bool bytes = a->x_dtype == ANSZP_I8;
    if ((!bytes && a->x_dtype != ANSZP_OUT_BF16) || (a->out_dtype != ANSZP_OUT_F32 && a->out_dtype != ANSZP_OUT_BF16) || a->activation > ANSZP_FN_SILU ||
        a->k == 0 || a->k > (bytes ? 65536u : 1u << 30) || a->rows >= 1ull << 31 || a->cols >= 1ull << 31 || a->zero_point > 255u)
        return ANSZP_E_RANGE;
    if (a->rows > 1 && a->out_stride < a->cols) return ANSZP_E_RANGE;
    if (a->rows == 0 || a->cols == 0) return ANSZP_OK;
    if (!a->x || !a->weight || !a->out) return ANSZP_E_NULL;
    const uint32_t size = bytes ? 1u : 2u;
    LinearParams p = {static_cast<const uint8_t*>(a->x), static_cast<const uint8_t*>(a->weight), a->x_scales, a->channel_scales, a->bias, a->mul, a->residual, a->out,
                      a->x_stride * size, a->weight_stride * size, a->mul_stride, a->residual_stride, a->out_stride, a->rows, a->cols,
                      a->k * size, a->activation, a->out_dtype, 128 - static_cast<int32_t>(a->zero_point), a->scale};
    const dim3 grid(static_cast<uint32_t>((p.cols + 63u) / 64u), static_cast<uint32_t>((p.rows + 63u) / 64u));
    if (grid.y > 65535u) return ANSZP_E_RANGE;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (bytes ? take_few<true>(p, s) : take_few<false>(p, s)) return hipGetLastError() == hipSuccess ? ANSZP_OK : ANSZP_E_HIP;
    if (bytes) hipLaunchKernelGGL(linear_any_kernel<true>, grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL(linear_any_kernel<false>, grid, dim3(256), 0, s, p);
    return hipGetLastError() == hipSuccess ? ANSZP_OK : ANSZP_E_HIP;
}
