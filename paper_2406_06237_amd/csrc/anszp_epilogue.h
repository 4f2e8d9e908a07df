// What products have behind their sums: activations, and operands of the output's type (internal to the library).
#ifndef ANSZP_EPILOGUE_H
#define ANSZP_EPILOGUE_H

#include "anszp_numbers.h"

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

#endif
