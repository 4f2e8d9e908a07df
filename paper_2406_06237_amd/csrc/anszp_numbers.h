// Number forms of the operators that run beside the decoded weights: bf16 and fp32 rows read eight elements at a time, results
// rounded to their type (internal to the library).
#ifndef ANSZP_NUMBERS_H
#define ANSZP_NUMBERS_H

#include <hip/hip_runtime.h>

#include <cstdint>
#include <utility>

#include "anszp.h"

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(4))) int32_t intx4;
typedef __attribute__((ext_vector_type(4))) uint32_t words4;
typedef __attribute__((ext_vector_type(2))) uint32_t words2;
// Rows begin at any element and widths are any number: loads and stores of 16 bytes are aligned to an element only, which global
// memory takes at full speed where they happen to be aligned.
typedef words4 __attribute__((aligned(1))) words4_any;
typedef words2 __attribute__((aligned(1))) words2_any;
typedef uint32_t __attribute__((aligned(1))) word_any;

__device__ __forceinline__ float bf16_low(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }
// to nearest, ties to even; a NaN stays one
__device__ __forceinline__ uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v)); }
__device__ __forceinline__ uint32_t to_bf16_pair(float a, float b) { return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a), static_cast<__bf16>(b)}); }

// Eight consecutive elements as they lie in memory; fewer where the row ends, the rest 0.
template <uint32_t DTYPE>
struct Eight;
template <>
struct Eight<ANSZP_OUT_BF16> {
    words4 w;
    __device__ __forceinline__ void load(const void* base, uint64_t at, uint32_t there) {
        const uint16_t* p = static_cast<const uint16_t*>(base) + at;
        w = words4{0u, 0u, 0u, 0u};
        if (there >= 8u) {
            w = *reinterpret_cast<const words4_any*>(p);
        } else {
            for (uint32_t i = 0; i < 8u; ++i)
                if (i < there) w[i >> 1] |= uint32_t(p[i]) << ((i & 1u) * 16u);
        }
    }
    __device__ __forceinline__ float operator[](uint32_t i) const { return i & 1u ? bf16_high(w[i >> 1]) : bf16_low(w[i >> 1]); }
};
template <>
struct Eight<ANSZP_OUT_F32> {
    words4 w[2];
    __device__ __forceinline__ void load(const void* base, uint64_t at, uint32_t there) {
        const uint32_t* p = static_cast<const uint32_t*>(base) + at;
        w[0] = w[1] = words4{0u, 0u, 0u, 0u};
        if (there >= 8u) {
            w[0] = *reinterpret_cast<const words4_any*>(p);
            w[1] = *reinterpret_cast<const words4_any*>(p + 4);
        } else {
            for (uint32_t i = 0; i < 8u; ++i)
                if (i < there) w[i >> 2][i & 3u] = p[i];
        }
    }
    __device__ __forceinline__ float operator[](uint32_t i) const {
        const uint32_t word = w[i >> 2][i & 3u];           // (a bit cast of the vector's element itself takes element 0)
        return __builtin_bit_cast(float, word);
    }
};

__device__ __forceinline__ void store_eight(void* base, uint32_t dtype, uint64_t at, uint32_t there, const float (&v)[8]) {
    if (dtype == ANSZP_OUT_BF16) {
        uint16_t* p = static_cast<uint16_t*>(base) + at;
        if (there >= 8u) {
            *reinterpret_cast<words4_any*>(p) = words4{to_bf16_pair(v[0], v[1]), to_bf16_pair(v[2], v[3]), to_bf16_pair(v[4], v[5]), to_bf16_pair(v[6], v[7])};
        } else {
            for (uint32_t i = 0; i < 8u; ++i)
                if (i < there) p[i] = to_bf16(v[i]);
        }
    } else {
        float* p = static_cast<float*>(base) + at;
        if (there >= 8u) {
            *reinterpret_cast<words4_any*>(p) = __builtin_bit_cast(words4, floatx4{v[0], v[1], v[2], v[3]});
            *reinterpret_cast<words4_any*>(p + 4) = __builtin_bit_cast(words4, floatx4{v[4], v[5], v[6], v[7]});
        } else {
            for (uint32_t i = 0; i < 8u; ++i)
                if (i < there) p[i] = v[i];
        }
    }
}

// A launch counts its threads in 32 bits in each dimension, and what is beyond is left out without an error: workgroups that can be more than that come in
// rows of kAcross (of up to 1024 threads each).
constexpr uint32_t kAcross = 1u << 21;
inline uint32_t groups_across(uint64_t groups) { return static_cast<uint32_t>(groups < kAcross ? groups : kAcross); }
inline uint32_t groups_down(uint64_t groups) { return static_cast<uint32_t>((groups + kAcross - 1u) / kAcross); }

// Rows of an operand, in bytes.
struct Rows {
    const void* at;
    uint64_t rows, stride, width;
};
// Whether two operands surely have memory in common.  (Rows of one may lie between the other's, as columns of one buffer do.  Of rows of two strides the first ones
// are looked at.)
inline bool meet(Rows a, Rows b) {
    if (!a.at || !b.at || a.rows == 0u || b.rows == 0u) return false;
    if (reinterpret_cast<uintptr_t>(b.at) < reinterpret_cast<uintptr_t>(a.at)) std::swap(a, b);
    if (a.rows == 1u) a.stride = a.width;
    if (b.rows == 1u) b.stride = b.width;
    const uint64_t apart = reinterpret_cast<uintptr_t>(b.at) - reinterpret_cast<uintptr_t>(a.at);
    if (apart >= (a.rows - 1u) * a.stride + a.width) return false;
    if (a.stride <= a.width) return true;
    const uint64_t row = apart / a.stride, behind = apart % a.stride, run = b.stride <= b.width ? (b.rows - 1u) * b.stride + b.width : b.width;
    return behind < a.width || (behind + run > a.stride && row + 1u < a.rows);
}
// ... though an output may be the operand itself, row for row.
inline bool meet_elsewhere(const Rows& out, const Rows& in) { return !(out.at == in.at && (out.rows <= 1u || out.stride == in.stride)) && meet(out, in); }

__device__ __forceinline__ uint64_t least(uint64_t a, uint64_t b) { return a < b ? a : b; }

#endif
