// Tokens looked up as rows, for gfx950: out[t] = scale * row_scales[id] * (w[id] - zero_point), the rows of a layer's symbols as anszp_decode leaves
// them (Sec. II-B), or of its values in bf16 (row_scales and zero_point have no part then).  One rounding to the output's type behind two in 32 bits.
//
// Memory bounds it: a lane has 16 elements of a row, which are 16 bytes of symbols, and rows lie wherever their token says.  16384 tokens of 4096 symbols take
// 32 us, 6.2 TB/s read and written; 16 tokens 2.8 us, three loads that wait for each other (token, row, and the row's scale).
#include <hip/hip_runtime.h>

#include "anszp_numbers.h"

namespace {

struct EmbedParams {
    const int64_t* tokens;
    const void* weight;
    const float* row_scales;
    void* out;
    uint32_t* status;
    uint64_t n_tokens, vocabulary, weight_stride, out_stride;
    uint32_t cols, pieces, out_dtype;   // pieces of 16 elements a row
    float zero_point, scale;
};

template <bool SYMBOLS>
__global__ __launch_bounds__(256) void embed_kernel(EmbedParams p) {
    const uint64_t n = (uint64_t(blockIdx.y) * kAcross + blockIdx.x) * 256u + threadIdx.x, t = n / p.pieces;
    if (t >= p.n_tokens) return;
    const uint32_t at = uint32_t(n - t * p.pieces) * 16u, there = p.cols - at < 16u ? p.cols - at : 16u;
    const int64_t id = p.tokens[t];
    float lo[8] = {}, hi[8] = {};
    if (uint64_t(id) < p.vocabulary) {
        const uint64_t from = uint64_t(id) * p.weight_stride + at;
        if constexpr (SYMBOLS) {
            const uint8_t* w = static_cast<const uint8_t*>(p.weight) + from;
            words4 q = {0u, 0u, 0u, 0u};
            if (there == 16u) {
                q = *reinterpret_cast<const words4_any*>(w);
            } else {
                for (uint32_t i = 0; i < 16u; ++i)
                    if (i < there) q[i >> 2] |= uint32_t(w[i]) << (8u * (i & 3u));
            }
            const float by = p.row_scales ? p.row_scales[id] * p.scale : p.scale;
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) {
                lo[i] = by * (float((q[i >> 2] >> (8u * (i & 3u))) & 0xFFu) - p.zero_point);
                hi[i] = by * (float((q[2u + (i >> 2)] >> (8u * (i & 3u))) & 0xFFu) - p.zero_point);
            }
        } else {
            Eight<ANSZP_OUT_BF16> a, b;
            a.load(p.weight, from, there);
            b.load(p.weight, from + 8u, there > 8u ? there - 8u : 0u);
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) {
                lo[i] = p.scale * a[i];
                hi[i] = p.scale * b[i];
            }
        }
    } else if (id >= 0 && at == 0u && p.status) {
        atomicOr(&p.status[0], ANSZP_ST_BAD_DESC);
        atomicAdd(&p.status[1], 1u);
    }
    store_eight(p.out, p.out_dtype, t * p.out_stride + at, there, lo);
    if (there > 8u) store_eight(p.out, p.out_dtype, t * p.out_stride + at + 8u, there - 8u, hi);
}

}  // namespace

extern "C" int anszp_embed(const anszp_embed_args_t* a, void* hip_stream) {
    if (!a) return ANSZP_E_NULL;
    const bool symbols = a->weight_dtype == ANSZP_OUT_U8;
    if ((!symbols && a->weight_dtype != ANSZP_OUT_BF16) || (a->out_dtype != ANSZP_OUT_F32 && a->out_dtype != ANSZP_OUT_BF16) || a->cols == 0 || a->cols >= 1u << 31 ||
        a->n_tokens >= 1ull << 31 || a->vocabulary >= 1ull << 31 || a->zero_point > (symbols ? 255u : 0u) || (!symbols && a->row_scales))
        return ANSZP_E_RANGE;
    if (a->n_tokens > 1 && a->out_stride < a->cols) return ANSZP_E_RANGE;
    if (a->n_tokens == 0) return ANSZP_OK;
    if (!a->tokens || !a->out || (a->vocabulary && !a->weight)) return ANSZP_E_NULL;
    const uint64_t size = a->out_dtype == ANSZP_OUT_BF16 ? 2u : 4u, weight_size = symbols ? 1u : 2u;
    const Rows out = {a->out, a->n_tokens, a->out_stride * size, a->cols * size};
    if (meet(out, {a->weight, a->vocabulary, a->weight_stride * weight_size, a->cols * weight_size}) || meet(out, {a->tokens, 1, 0, a->n_tokens * 8u}) ||
        meet(out, {a->row_scales, 1, 0, a->vocabulary * 4u}))
        return ANSZP_E_RANGE;
    EmbedParams p = {a->tokens, a->weight, a->row_scales, a->out, a->status, a->n_tokens, a->vocabulary, a->weight_stride, a->out_stride, a->cols, (a->cols + 15u) / 16u,
                     a->out_dtype, static_cast<float>(a->zero_point), a->scale};
    const uint64_t groups = (a->n_tokens * p.pieces + 255u) / 256u;
    if (groups_down(groups) > 65535u) return ANSZP_E_RANGE;
    const dim3 grid(groups_across(groups), groups_down(groups));
    if (symbols) hipLaunchKernelGGL(embed_kernel<true>, grid, dim3(256), 0, static_cast<hipStream_t>(hip_stream), p);
    else hipLaunchKernelGGL(embed_kernel<false>, grid, dim3(256), 0, static_cast<hipStream_t>(hip_stream), p);
    return hipGetLastError() == hipSuccess ? ANSZP_OK : ANSZP_E_HIP;
}
