// Root-mean-square norm of rows with the residual's addition, in fp32, bf16 or 8 bits, for gfx950:
//   h = x + r            y = h * (mean(h^2) + eps)^(-1/2) * g
//   s = max|y| / 127     q = round(y / s)                          (8 bits: a scale for each row)
// A row is read once and kept in registers; its sum of squares and max|h * g| are found in the same pass, since
//   max|y| = max|h * g| * (mean(h^2) + eps)^(-1/2)    and    y / s = h * g * 127 / max|h * g|,
// so that a row costs one exchange between its wavefronts.  Sums and products are held in 32 bits; what is rounded is h to x's
// type where the sum is asked for (the norm goes on with h itself) and y to the output's.
// Memory bounds it: 4096 rows of 4096 in bfloat16 with a residual, its sum and 8 bits out take 22 us, 5.3 TB/s of what is read and written (a large copy
// reaches 4.8); one row takes 3 us, which is an empty launch's time.
#include <hip/hip_runtime.h>

#include "anszp_numbers.h"

namespace {

struct NormParams {
    const void* x;
    const void* residual;
    void* total;
    const void* weight;
    void* out;
    float* out_scales;
    uint64_t rows, x_stride, residual_stride, total_stride, out_stride;
    uint32_t cols, out_dtype, weight_dtype, normalise;
    float eps, inverse_cols;
};

struct Gathered {
    float squares, most, poison;
};

__device__ __forceinline__ Gathered over_wave(Gathered g) {
    for (int d = 32; d; d >>= 1) {
        g.squares += __shfl_xor(g.squares, d);
        g.most = fmaxf(g.most, __shfl_xor(g.most, d));
        g.poison += __shfl_xor(g.poison, d);
    }
    return g;
}

// of all THREADS threads of a row; wavefronts that have a row each have nothing to exchange
template <uint32_t THREADS>
__device__ __forceinline__ Gathered over_row(Gathered g) {
    g = over_wave(g);
    if constexpr (THREADS > 64u) {
        __shared__ Gathered of_wave[THREADS / 64u];
        if ((threadIdx.x & 63u) == 0u) of_wave[threadIdx.x >> 6] = g;
        __syncthreads();
        g = of_wave[0];
        for (uint32_t w = 1; w < THREADS / 64u; ++w) {
            g.squares += of_wave[w].squares;
            g.most = fmaxf(g.most, of_wave[w].most);
            g.poison += of_wave[w].poison;
        }
    }
    return g;
}

__device__ __forceinline__ void weights_of(const NormParams& p, uint32_t at, uint32_t there, float (&g)[8]) {
    if (p.weight_dtype == ANSZP_OUT_BF16) {
        Eight<ANSZP_OUT_BF16> w;
        w.load(p.weight, at, there);
        for (uint32_t i = 0; i < 8u; ++i) g[i] = w[i];
    } else {
        Eight<ANSZP_OUT_F32> w;
        w.load(p.weight, at, there);
        for (uint32_t i = 0; i < 8u; ++i) g[i] = w[i];
    }
}

// What takes h * g to what is stored: times `factor`, or with 8 bits of a row near binary32's least numbers, where 127 / max|h * g| is more than 32 bits
// hold, times 2^64 before.
struct Factor {
    float factor;
    bool tiny;
};
constexpr float kLift = 0x1p64f;

// h * g on: times the row's factor, rounded and stored.
__device__ __forceinline__ void store_row_part(const NormParams& p, uint64_t row, uint32_t at, uint32_t there, const float (&y)[8], const Factor& by) {
    float v[8];
    for (uint32_t i = 0; i < 8u; ++i) v[i] = y[i] * by.factor;
    const uint64_t to = row * p.out_stride + at;
    if (p.out_dtype != ANSZP_I8) {
        store_eight(p.out, p.out_dtype, to, there, v);
        return;
    }
    if (by.tiny)
        for (uint32_t i = 0; i < 8u; ++i) v[i] = __builtin_amdgcn_fmed3f(y[i] * kLift * by.factor, -127.0f, 127.0f);    // (the scale may have been rounded down)
    words2 q = {0u, 0u};
    for (uint32_t i = 0; i < 8u; ++i) q[i >> 2] |= (uint32_t(int32_t(rintf(v[i]))) & 0xFFu) << (8u * (i & 3u));
    int8_t* out = static_cast<int8_t*>(p.out) + to;
    if (there >= 8u) {
        *reinterpret_cast<words2_any*>(out) = q;
    } else {
        for (uint32_t i = 0; i < 8u; ++i)
            if (i < there) out[i] = static_cast<int8_t>(q[i >> 2] >> (8u * (i & 3u)));
    }
}

// 8 bits: 127 / max|h * g|.  A row with an infinity or a NaN, in h * g or behind the norm, has no 8-bit form: its scale is NaN, its symbols 0.  Where the scale or
// the largest h * g is near binary32's least numbers (below 2^-100), the symbols are y over the scale as it is stored, which may have few bits left.
__device__ __forceinline__ Factor row_factor(const NormParams& p, const Gathered& g, uint64_t row, bool writes) {
    const float norm = p.normalise ? 1.0f / sqrtf(g.squares * p.inverse_cols + p.eps) : 1.0f;
    if (p.out_dtype != ANSZP_I8) return {norm, false};
    const bool sound = g.poison == 0.0f && g.most * norm < __builtin_inff();
    float scale = g.most * norm * (1.0f / 127.0f), factor = sound && g.most > 0.0f ? 127.0f / g.most : 0.0f;
    const bool tiny = sound && g.most < 1.0f && fminf(scale, g.most) < 0x1p-100f;
    if (tiny) {
        scale = g.most * kLift * norm * (1.0f / 127.0f) * (1.0f / kLift);
        factor = scale > 0.0f ? norm / (scale * kLift) : 0.0f;
    }
    if (writes) p.out_scales[row] = sound ? scale : __builtin_nanf("");
    return {factor, tiny};
}

// Rows of at most 8 * NV * THREADS elements.  Workgroups of several wavefronts have a row, or (THREADS = 64) each wavefront has one.
template <uint32_t DTYPE, uint32_t THREADS, uint32_t NV>
__global__ __launch_bounds__(THREADS == 64u ? 256u : THREADS) void rms_norm_kernel(NormParams p) {
    const uint32_t t = THREADS == 64u ? threadIdx.x & 63u : threadIdx.x;
    const uint64_t group = uint64_t(blockIdx.y) * kAcross + blockIdx.x, row = THREADS == 64u ? group * 4u + (threadIdx.x >> 6) : group;
    if (row >= p.rows) return;
    Eight<DTYPE> x[NV], r[NV];
    float g[NV][8];
    for (uint32_t v = 0; v < NV; ++v) {
        const uint32_t at = (v * THREADS + t) * 8u, there = at < p.cols ? p.cols - at : 0u;
        x[v].load(p.x, row * p.x_stride + at, there);
        if (p.residual) r[v].load(p.residual, row * p.residual_stride + at, there);
        if (p.normalise) weights_of(p, at, there, g[v]);
    }
    Gathered mine = {0.0f, 0.0f, 0.0f};
    for (uint32_t v = 0; v < NV; ++v) {
        const uint32_t at = (v * THREADS + t) * 8u, there = at < p.cols ? p.cols - at : 0u;
        float h[8];
        for (uint32_t i = 0; i < 8u; ++i) {
            h[i] = x[v][i];
            if (p.residual) h[i] += r[v][i];
            mine.squares = fmaf(h[i], h[i], mine.squares);
            mine.poison = fmaf(h[i], 0.0f, mine.poison);
            const float y = p.normalise ? h[i] * g[v][i] : h[i];
            mine.poison = fmaf(y, 0.0f, mine.poison);
            mine.most = fmaxf(mine.most, fabsf(y));
            g[v][i] = y;
        }
        if (p.total) store_eight(p.total, DTYPE, row * p.total_stride + at, there, h);
    }
    const Factor factor = row_factor(p, over_row<THREADS>(mine), row, t == 0u);
    for (uint32_t v = 0; v < NV; ++v) {
        const uint32_t at = (v * THREADS + t) * 8u;
        if (at < p.cols) store_row_part(p, row, at, p.cols - at, g[v], factor);
    }
}

// Longer rows are read twice.  What is written over an input is written when the thread has read it for the last time.
template <uint32_t DTYPE>
__global__ __launch_bounds__(1024) void rms_norm_long_kernel(NormParams p) {
    const uint64_t row = uint64_t(blockIdx.y) * kAcross + blockIdx.x;
    if (row >= p.rows) return;
    Gathered mine = {0.0f, 0.0f, 0.0f};
    Factor factor = {0.0f, false};
    for (uint32_t pass = 0; pass < 2u; ++pass) {
        for (uint64_t from = threadIdx.x * 8u; from < p.cols; from += 8192u) {
            const uint32_t at = uint32_t(from), there = p.cols - at;
            Eight<DTYPE> x, r;
            float h[8], y[8];
            x.load(p.x, row * p.x_stride + at, there);
            if (p.residual) r.load(p.residual, row * p.residual_stride + at, there);
            if (p.normalise) weights_of(p, at, there, y);
            for (uint32_t i = 0; i < 8u; ++i) {
                h[i] = x[i];
                if (p.residual) h[i] += r[i];
                y[i] = p.normalise ? h[i] * y[i] : h[i];
                if (pass == 0u) {
                    mine.squares = fmaf(h[i], h[i], mine.squares);
                    mine.poison = fmaf(h[i], 0.0f, fmaf(y[i], 0.0f, mine.poison));
                    mine.most = fmaxf(mine.most, fabsf(y[i]));
                }
            }
            if (pass == 1u) {
                if (p.total) store_eight(p.total, DTYPE, row * p.total_stride + at, there, h);
                store_row_part(p, row, at, there, y, factor);
            }
        }
        if (pass == 0u) factor = row_factor(p, over_row<1024u>(mine), row, threadIdx.x == 0u);
    }
}

template <uint32_t DTYPE>
void launch(const NormParams& p, hipStream_t s) {
    const uint32_t eights = (p.cols + 7u) / 8u;
    const dim3 rows(groups_across(p.rows), groups_down(p.rows)), fours(groups_across((p.rows + 3u) / 4u), groups_down((p.rows + 3u) / 4u));
    if (eights <= 64u) hipLaunchKernelGGL((rms_norm_kernel<DTYPE, 64u, 1u>), fours, dim3(256), 0, s, p);
    else if (eights <= 128u) hipLaunchKernelGGL((rms_norm_kernel<DTYPE, 64u, 2u>), fours, dim3(256), 0, s, p);
    else if (eights <= 256u) hipLaunchKernelGGL((rms_norm_kernel<DTYPE, 256u, 1u>), rows, dim3(256), 0, s, p);
    else if (eights <= 512u) hipLaunchKernelGGL((rms_norm_kernel<DTYPE, 256u, 2u>), rows, dim3(256), 0, s, p);
    else if (eights <= 1024u) hipLaunchKernelGGL((rms_norm_kernel<DTYPE, 512u, 2u>), rows, dim3(512), 0, s, p);
    else if (eights <= 2048u) hipLaunchKernelGGL((rms_norm_kernel<DTYPE, 1024u, 2u>), rows, dim3(1024), 0, s, p);
    else hipLaunchKernelGGL((rms_norm_long_kernel<DTYPE>), rows, dim3(1024), 0, s, p);
}

}  // namespace

extern "C" int anszp_rms_norm(const anszp_norm_args_t* a, void* hip_stream) {
    if (!a) return ANSZP_E_NULL;
    const bool eight_bits = a->out_dtype == ANSZP_I8;
    if ((a->dtype != ANSZP_OUT_F32 && a->dtype != ANSZP_OUT_BF16) || (a->out_dtype != ANSZP_OUT_F32 && a->out_dtype != ANSZP_OUT_BF16 && !eight_bits) ||
        (a->normalise && a->weight_dtype != ANSZP_OUT_F32 && a->weight_dtype != ANSZP_OUT_BF16) || a->cols == 0 || a->cols >= 1u << 31 || a->rows >= 1ull << 31)
        return ANSZP_E_RANGE;
    if (a->rows > 1 && (a->out_stride < a->cols || (a->total && a->total_stride < a->cols))) return ANSZP_E_RANGE;
    if (a->rows == 0) return ANSZP_OK;
    if (!a->x || !a->out || (a->normalise && !a->weight) || (eight_bits && !a->out_scales)) return ANSZP_E_NULL;
    const uint64_t size = a->dtype == ANSZP_OUT_BF16 ? 2u : 4u, out_size = eight_bits ? 1u : a->out_dtype == ANSZP_OUT_BF16 ? 2u : 4u, width = a->cols * size;
    const Rows out = {a->out, a->rows, a->out_stride * out_size, a->cols * out_size}, total = {a->total, a->rows, a->total_stride * size, width};
    const Rows x = {a->x, a->rows, a->x_stride * size, width}, residual = {a->residual, a->rows, a->residual_stride * size, width};
    if (meet(out, x) || meet(out, residual) || meet(out, total) || meet_elsewhere(total, x) || meet_elsewhere(total, residual)) return ANSZP_E_RANGE;
    NormParams p = {a->x, a->residual, a->total, a->weight, a->out, a->out_scales, a->rows, a->x_stride, a->residual_stride, a->total_stride, a->out_stride,
                    a->cols, a->out_dtype, a->weight_dtype, a->normalise ? 1u : 0u, a->eps, 1.0f / static_cast<float>(a->cols)};
    if (a->dtype == ANSZP_OUT_F32) launch<ANSZP_OUT_F32>(p, static_cast<hipStream_t>(hip_stream));
    else launch<ANSZP_OUT_BF16>(p, static_cast<hipStream_t>(hip_stream));
    return hipGetLastError() == hipSuccess ? ANSZP_OK : ANSZP_E_HIP;
}
