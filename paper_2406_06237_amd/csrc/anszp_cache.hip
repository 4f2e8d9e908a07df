// Keys and values quantised as they are written to a paged cache, and read back, for gfx950.  A vector is one head's key or value
// of one token; it has a scale and a zero-point of its own, in the form of Sec. II-B, w = scale * (q - zero_point):
//   lo = min(0, min x)   hi = max(0, max x)   scale = (hi - lo) * (1 / (2^bits - 1))
//   zero_point = round(-lo / scale)           q = clamp(round(x / scale) + zero_point, 0, 2^bits - 1)
// with every operation rounded to binary32 (the reciprocal too; ties to even throughout), so that any program that follows the
// formulas finds the same symbols: elements of few bits stand halfway between two symbols often.  0 is always a symbol's value, as Sec. II-B asks of a zero-point.
//
// Memory is what bounds both kernels: a lane has 8 elements, head_dim / 8 lanes a vector, so that 16 bytes in and 8 (or 4) bytes
// out per lane lie one behind the other; the vector's extremes are found in log2(head_dim / 8) exchanges between those lanes.
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
    uint32_t heads, page_log, dim;
};

// What a vector's number stands for.  In device memory a page has [head][token in page][symbols].
struct Place {
    uint64_t token;
    uint32_t head;
    uint64_t vector;                    // index of the vector in the cache
    bool there;
};

__device__ __forceinline__ Place place_of(const CacheParams& p, uint64_t n, bool first_lane) {
    Place at;
    if (n >> 32) {
        at.token = n / p.heads;
        at.head = uint32_t(n - at.token * p.heads);
    } else {
        const uint32_t token = uint32_t(n) / p.heads;
        at.token = token;
        at.head = uint32_t(n) - token * p.heads;
    }
    const int64_t slot = p.slots[at.token];
    at.there = slot >= 0 && uint64_t(slot) < p.n_slots;
    if (slot >= 0 && !at.there && first_lane && at.head == 0u && blockIdx.y == 0u && p.status) {
        atomicOr(&p.status[0], ANSZP_ST_BAD_DESC);
        atomicAdd(&p.status[1], 1u);
    }
    const uint64_t s = at.there ? uint64_t(slot) : 0u;
    at.vector = (((s >> p.page_log) * p.heads + at.head) << p.page_log) + (s & ((1ull << p.page_log) - 1u));
    return at;
}

template <uint32_t DTYPE, uint32_t BITS>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheParams p) {
    const uint32_t lanes = p.dim / 8u;                              // 8, 16 or 32
    const uint32_t which = blockIdx.y;
    const uint64_t thread = uint64_t(blockIdx.x) * 256u + threadIdx.x;
    const uint32_t lane = threadIdx.x & (lanes - 1u);
    const uint64_t n = thread / lanes;
    if (n >= p.vectors) return;                                     // (whole vectors of lanes leave)
    const Place at = place_of(p, n, lane == 0u);
    if (!at.there) return;
    Eight<DTYPE> x;
    x.load(p.in[which], at.token * p.token_stride[which] + at.head * p.head_stride[which] + lane * 8u, 8u);
    float lo = 0.0f, hi = 0.0f, poison = 0.0f;
    for (uint32_t i = 0; i < 8u; ++i) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
        poison = fmaf(x[i], 0.0f, poison);
    }
    for (uint32_t d = lanes / 2u; d; d >>= 1) {
        lo = fminf(lo, __shfl_xor(lo, d));
        hi = fmaxf(hi, __shfl_xor(hi, d));
        poison += __shfl_xor(poison, d);
    }
    constexpr float kMost = float((1u << BITS) - 1u);
    float scale = (hi - lo) * (1.0f / kMost);
    const bool sound = poison == 0.0f && scale < __builtin_inff();
    const float by = sound && scale > 0.0f ? scale : 1.0f;          // (a range below what 32 bits can divide is all zero-point)
    const float zero = sound && scale > 0.0f ? rintf(-lo / by) : 0.0f;
    uint32_t q[8];
    if (by >= 0x1p-100f && by <= 0x1p100f) {
        // x / by rounded once, in three instructions: y the reciprocal rounded, a = x y rounded, then a + (x - a by) y is x / by rounded (Markstein's
        // theorem; away from the ends of the exponents' range, where no quotient that matters here lies).
        const float y = 1.0f / by;
        for (uint32_t i = 0; i < 8u; ++i) {
            const float a = x[i] * y;
            q[i] = uint32_t(fminf(fmaxf(rintf(fmaf(fmaf(-a, by, x[i]), y, a)) + zero, 0.0f), kMost));
        }
    } else {
        for (uint32_t i = 0; i < 8u; ++i) q[i] = uint32_t(fminf(fmaxf(rintf(x[i] / by) + zero, 0.0f), kMost));
    }
    if (!(sound && scale > 0.0f))
        for (uint32_t i = 0; i < 8u; ++i) q[i] = 0u;
    uint8_t* to = p.symbols[which] + at.vector * (p.dim * BITS / 8u);
    if constexpr (BITS == 8u)
        reinterpret_cast<words2*>(to)[lane] = words2{q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24, q[4] | q[5] << 8 | q[6] << 16 | q[7] << 24};
    else
        reinterpret_cast<uint32_t*>(to)[lane] = q[0] | q[1] << 4 | q[2] << 8 | q[3] << 12 | q[4] << 16 | q[5] << 20 | q[6] << 24 | q[7] << 28;
    if (lane == 0u) reinterpret_cast<float2*>(p.params[which])[at.vector] = make_float2(sound ? scale : __builtin_nanf(""), zero);
}

template <uint32_t BITS>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheParams p, uint32_t out_dtype) {
    const uint32_t lanes = p.dim / 8u;
    const uint32_t which = blockIdx.y;
    const uint64_t thread = uint64_t(blockIdx.x) * 256u + threadIdx.x;
    const uint32_t lane = threadIdx.x & (lanes - 1u);
    const uint64_t n = thread / lanes;
    if (n >= p.vectors) return;
    const Place at = place_of(p, n, lane == 0u);
    float v[8] = {};
    if (at.there) {
        const uint8_t* from = p.symbols[which] + at.vector * (p.dim * BITS / 8u);
        const float2 w = reinterpret_cast<const float2*>(p.params[which])[at.vector];
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
    return p.vectors * (c->head_dim / 8u) / 256u >= 1ull << 31 ? ANSZP_E_RANGE : ANSZP_OK;
}

dim3 grid_of(const CacheParams& p) { return dim3(static_cast<uint32_t>((p.vectors * (p.dim / 8u) + 255u) / 256u), 2); }

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
