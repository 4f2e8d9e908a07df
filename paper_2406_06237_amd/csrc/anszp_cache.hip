// Keys and values quantised as they are written to a paged cache, and read back, for gfx950.  A vector is one head's key or value
// of one token; it has a scale and a zero-point of its own, in the form of Sec. II-B, w = scale * (q - zero_point):
//   lo = min(0, min x)   hi = max(0, max x)   scale = (hi - lo) * (1 / (2^bits - 1))
//   zero_point = round(-lo / scale)           q = clamp(round(x / scale) + zero_point, 0, 2^bits - 1)
// with every operation rounded to binary32 (the reciprocal too; ties to even throughout), so that any program that follows the
// formulas finds the same symbols: elements of few bits stand halfway between two symbols often.  0 is always a symbol's value, as Sec. II-B asks of a zero-point.
//
// Memory is what bounds both kernels, and instructions nearly: a lane has 8 elements, head_dim / 8 lanes a vector, so that 16 bytes in and 8 (or 4)
// bytes out per lane lie one behind the other; the vector's extremes are found in log2(head_dim / 8) exchanges between those lanes.  8191 tokens
// of 32 heads of 128 in bfloat16, keys and values, 4 bits: written in 46 us and read back in 35, 4.25 TB/s of what both read and write (a large copy
// reaches 4.83).  (The writing took 57 us while the elements were asked for behind their slot's check, the exchanges went through LDS and symbols were
// packed one shift at a time.)  16 tokens of the same, 8 bits, take 3.1 and 3.0 us, which is an empty launch's time.
#include <hip/hip_runtime.h>

#include "anszp_numbers.h"

namespace {

struct CacheParams {
    uint8_t* symbols[2];                // keys, values
    float* params[2];
    const void* in[2];
    void* out[2];
    const int64_t* slots;
    uint32_t* status;
    uint64_t n_slots, vectors;          // tokens * heads
    uint64_t token_stride[2], head_stride[2];
    uint32_t heads, page_log, dim, lanes_log;   // lanes of a vector: dim / 8
};

// What a vector's number stands for.
struct Vector {
    uint64_t token;
    uint32_t head;
};
__device__ __forceinline__ Vector vector_of(const CacheParams& p, uint64_t n) {
    if (p.vectors >> 32) {
        const uint64_t token = n / p.heads;
        return {token, uint32_t(n - token * p.heads)};
    }
    const uint32_t token = uint32_t(n) / p.heads;
    return {token, uint32_t(n) - token * p.heads};
}

// Where a token's slot puts it: a page has [head][token in page][symbols].
__device__ __forceinline__ bool there(const CacheParams& p, int64_t slot, const Vector& v, bool first_lane) {
    if (uint64_t(slot) < p.n_slots) return true;
    if (slot >= 0 && first_lane && v.head == 0u && blockIdx.y == 0u && p.status) {
        atomicOr(&p.status[0], ANSZP_ST_BAD_DESC);
        atomicAdd(&p.status[1], 1u);
    }
    return false;
}
__device__ __forceinline__ uint64_t place_of(const CacheParams& p, uint64_t slot, uint32_t head) {
    return (((slot >> p.page_log) * p.heads + head) << p.page_log) + (slot & ((1ull << p.page_log) - 1u));
}

// The largest of `v` over the lanes of a vector, 8, 16 or 32 of them.  (Lanes trade by their place in a row of 16 as operands, without LDS.)
template <int CONTROL>
__device__ __forceinline__ float traded(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CONTROL, 0xF, 0xF, true));
}
__device__ __forceinline__ float largest(float v, uint32_t lanes) {
    v = fmaxf(v, traded<0xB1>(v));                                  // quad_perm [1, 0, 3, 2]
    v = fmaxf(v, traded<0x4E>(v));                                  // quad_perm [2, 3, 0, 1]
    v = fmaxf(v, traded<0x141>(v));                                 // a half row mirrored
    if (lanes > 8u) v = fmaxf(v, traded<0x140>(v));                 // a row mirrored
    if (lanes > 16u) v = fmaxf(v, __shfl_xor(v, 16));
    return v;
}

template <uint32_t DTYPE, uint32_t BITS>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheParams p) {
    const uint32_t lanes = 1u << p.lanes_log;                       // 8, 16 or 32
    const uint32_t which = blockIdx.y;
    const uint32_t lane = threadIdx.x & (lanes - 1u);
    const uint64_t n = ((uint64_t(blockIdx.z) * kAcross + blockIdx.x) * 256u + threadIdx.x) >> p.lanes_log;
    if (n >= p.vectors) return;                                     // (whole vectors of lanes leave)
    const Vector at = vector_of(p, n);
    int64_t slot = p.slots[at.token];
    Eight<DTYPE> x;
    x.load(p.in[which], at.token * p.token_stride[which] + at.head * p.head_stride[which] + lane * 8u, 8u);
    asm volatile("" : "+v"(slot) : "v"(x[0]));                      // (both are under way together: a slot that is none is rare)
    if (!there(p, slot, at, lane == 0u)) return;
    const uint64_t place = place_of(p, uint64_t(slot), at.head);
    float lo = 0.0f, hi = 0.0f, poison = 0.0f;
    for (uint32_t i = 0; i < 8u; ++i) {
        lo = fmaxf(lo, -x[i]);
        hi = fmaxf(hi, x[i]);
        poison = fmaf(x[i], 0.0f, poison);
    }
    hi = poison == 0.0f ? hi : __builtin_inff();                    // infinity and NaN: no finite scale
    lo = -largest(lo, lanes);
    hi = largest(hi, lanes);
    constexpr float kMost = float((1u << BITS) - 1u);
    float scale = (hi - lo) * (1.0f / kMost);
    const bool sound = scale < __builtin_inff();
    const float by = sound && scale > 0.0f ? scale : 1.0f;          // (a range below what 32 bits can divide is all zero-point)
    const float zero = sound && scale > 0.0f ? rintf(-lo / by) : 0.0f;
    float f[8];
    if (by >= 0x1p-100f && by <= 0x1p100f) {
        // x / by rounded once, in three instructions: y the reciprocal rounded, a = x y rounded, then a + (x - a by) y is x / by rounded (Markstein's
        // theorem; away from the ends of the exponents' range, where no quotient that matters here lies).
        const float y = 1.0f / by;
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) {
            const float a = x[i] * y;
            f[i] = fmaf(fmaf(-a, by, x[i]), y, a);
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) f[i] = x[i] / by;
    }
    const bool any = sound && scale > 0.0f;
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) f[i] = any ? __builtin_amdgcn_fmed3f(rintf(f[i]) + zero, 0.0f, kMost) : 0.0f;
    uint8_t* to = p.symbols[which] + place * (p.dim * BITS / 8u);
    if constexpr (BITS == 8u) {
        words2 w = {0u, 0u};
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) w[i >> 2] = __builtin_amdgcn_cvt_pk_u8_f32(f[i], i & 3u, w[i >> 2]);
        reinterpret_cast<words2*>(to)[lane] = w;
    } else {
        uint32_t w = 0u;                                            // two symbols' byte is a whole number below 256
#pragma unroll
        for (uint32_t i = 0; i < 4u; ++i) w = __builtin_amdgcn_cvt_pk_u8_f32(fmaf(f[2u * i + 1u], 16.0f, f[2u * i]), i, w);
        reinterpret_cast<uint32_t*>(to)[lane] = w;
    }
    if (lane == 0u) reinterpret_cast<float2*>(p.params[which])[place] = make_float2(sound ? scale : __builtin_nanf(""), zero);
}

template <uint32_t BITS>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheParams p, uint32_t out_dtype) {
    const uint32_t which = blockIdx.y;
    const uint32_t lane = threadIdx.x & ((1u << p.lanes_log) - 1u);
    const uint64_t n = ((uint64_t(blockIdx.z) * kAcross + blockIdx.x) * 256u + threadIdx.x) >> p.lanes_log;
    if (n >= p.vectors) return;
    const Vector at = vector_of(p, n);
    const int64_t slot = p.slots[at.token];
    float v[8] = {};
    if (there(p, slot, at, lane == 0u)) {
        const uint64_t place = place_of(p, uint64_t(slot), at.head);
        const uint8_t* from = p.symbols[which] + place * (p.dim * BITS / 8u);
        const float2 w = reinterpret_cast<const float2*>(p.params[which])[place];
        words2 q;
        if constexpr (BITS == 8u) {
            q = reinterpret_cast<const words2*>(from)[lane];
            for (uint32_t i = 0; i < 8u; ++i) v[i] = w.x * (float((q[i >> 2] >> (8u * (i & 3u))) & 0xFFu) - w.y);
        } else {
            q[0] = reinterpret_cast<const uint32_t*>(from)[lane];
            for (uint32_t i = 0; i < 8u; ++i) v[i] = w.x * (float((q[0] >> (4u * i)) & 15u) - w.y);
        }
    }
    store_eight(p.out[which], out_dtype, n * p.dim + lane * 8u, 8u, v);
}

// The checks both calls share, and the parameters.
int cache_params(const anszp_cache_t* c, const int64_t* slots, uint64_t n_tokens, uint32_t* status, CacheParams& p) {
    if (!c) return ANSZP_E_NULL;
    const int rc = anszp_cache_check(c);
    if (rc) return rc;
    if (n_tokens >= 1ull << 31) return ANSZP_E_RANGE;
    if (n_tokens && !slots) return ANSZP_E_NULL;
    p.symbols[0] = c->k; p.symbols[1] = c->v;
    p.params[0] = c->k_params; p.params[1] = c->v_params;
    p.slots = slots;
    p.status = status;
    p.n_slots = c->n_pages * c->page_size;
    p.vectors = n_tokens * c->heads;
    p.heads = c->heads;
    p.page_log = static_cast<uint32_t>(__builtin_ctz(c->page_size));
    p.dim = c->head_dim;
    p.lanes_log = static_cast<uint32_t>(__builtin_ctz(c->head_dim / 8u));
    return p.vectors * (c->head_dim / 8u) / 256u >= 1ull << 31 ? ANSZP_E_RANGE : ANSZP_OK;
}

dim3 grid_of(const CacheParams& p) {
    const uint64_t groups = (p.vectors * (p.dim / 8u) + 255u) / 256u;
    return dim3(groups_across(groups), 2, groups_down(groups));
}

}  // namespace

extern "C" {

int anszp_cache_check(const anszp_cache_t* c) {
    if (!c) return ANSZP_E_NULL;
    if (c->page_size < 16u || c->page_size > 65536u || (c->page_size & (c->page_size - 1u)) || c->heads == 0u || c->heads > 65535u ||
        (c->head_dim != 64u && c->head_dim != 128u && c->head_dim != 256u) || (c->bits != 8u && c->bits != 4u) || c->n_pages >= 1ull << 31 ||
        c->n_pages * c->heads >= (1ull << 32) / c->page_size)            // (no GPU has memory for 2^32 vectors)
        return ANSZP_E_RANGE;
    if (c->n_pages && (!c->k || !c->v || !c->k_params || !c->v_params)) return ANSZP_E_NULL;
    if ((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v)) & 15u) return ANSZP_E_RANGE;
    if ((reinterpret_cast<uintptr_t>(c->k_params) | reinterpret_cast<uintptr_t>(c->v_params)) & 15u) return ANSZP_E_RANGE;
    return ANSZP_OK;
}

int anszp_cache_write(const anszp_cache_t* cache, const void* k, const void* v, uint32_t dtype, uint64_t k_token_stride, uint64_t k_head_stride,
                      uint64_t v_token_stride, uint64_t v_head_stride, const int64_t* slots, uint64_t n_tokens, uint32_t* status, void* hip_stream) {
    CacheParams p = {};
    const int rc = cache_params(cache, slots, n_tokens, status, p);
    if (rc) return rc;
    if (dtype != ANSZP_OUT_F32 && dtype != ANSZP_OUT_BF16) return ANSZP_E_RANGE;
    if (n_tokens == 0) return ANSZP_OK;
    if (!k || !v) return ANSZP_E_NULL;
    p.in[0] = k; p.in[1] = v;
    p.token_stride[0] = k_token_stride; p.token_stride[1] = v_token_stride;
    p.head_stride[0] = k_head_stride; p.head_stride[1] = v_head_stride;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (dtype == ANSZP_OUT_F32) {
        if (cache->bits == 8u) hipLaunchKernelGGL((cache_write_kernel<ANSZP_OUT_F32, 8u>), grid_of(p), dim3(256), 0, s, p);
        else hipLaunchKernelGGL((cache_write_kernel<ANSZP_OUT_F32, 4u>), grid_of(p), dim3(256), 0, s, p);
    } else {
        if (cache->bits == 8u) hipLaunchKernelGGL((cache_write_kernel<ANSZP_OUT_BF16, 8u>), grid_of(p), dim3(256), 0, s, p);
        else hipLaunchKernelGGL((cache_write_kernel<ANSZP_OUT_BF16, 4u>), grid_of(p), dim3(256), 0, s, p);
    }
    return hipGetLastError() == hipSuccess ? ANSZP_OK : ANSZP_E_HIP;
}

int anszp_cache_read(const anszp_cache_t* cache, void* k, void* v, uint32_t dtype, const int64_t* slots, uint64_t n_tokens, uint32_t* status, void* hip_stream) {
    CacheParams p = {};
    const int rc = cache_params(cache, slots, n_tokens, status, p);
    if (rc) return rc;
    if (dtype != ANSZP_OUT_F32 && dtype != ANSZP_OUT_BF16) return ANSZP_E_RANGE;
    if (n_tokens == 0) return ANSZP_OK;
    if (!k || !v) return ANSZP_E_NULL;
    p.out[0] = k; p.out[1] = v;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (cache->bits == 8u) hipLaunchKernelGGL(cache_read_kernel<8u>, grid_of(p), dim3(256), 0, s, p, dtype);
    else hipLaunchKernelGGL(cache_read_kernel<4u>, grid_of(p), dim3(256), 0, s, p, dtype);
    return hipGetLastError() == hipSuccess ? ANSZP_OK : ANSZP_E_HIP;
}

}  // extern "C"
