// Attention of new tokens over the quantised paged cache, for gfx950:
//   out = sum_t softmax_t(scale * q . k_t) v_t,      k_t = s_t (symbol - z_t),  v_t alike.
// One pass over the tokens with the running maximum m and sum l of each query's weights, 32 tokens a step, products in
// v_mfma_f32_16x16x32_f16.  The rows of a tile are the queries of one head of the cache: (new token, query head of the group).
//
// Symbols become matrix operands in registers, without conversions and exactly: fp16 holds 1024 + q for every byte q as the bits 0x6400 | q, so that
// symbol - z is a byte permutation and a packed subtraction of 1024 + z; values get by with a permutation and a packed multiplication and addition
// (value_pair).  A key's scale multiplies its scores; a value's scale goes into the weight.
//   scores^T = K Q^T: lane (c, g), c = lane % 16, g = lane / 16, feeds a key's dimensions [g D / 4, (g + 1) D / 4), which lie one behind
//     the other in memory, and ends up with the scores of query c for tokens 4 g .. 4 g + 3 of each half of the step;
//   out^T = V^T P^T: those are the weights the lane has to feed for query c, so they never leave their lane.  It feeds, for the same tokens,
//     the dimensions [c D / 16, (c + 1) D / 16) of their values, 16 lanes reading a value end to end, and the bytes of one dimension
//     are brought together by v_perm_b32.  Nothing passes through LDS but the join of the wavefronts' results.
// Queries are scaled per row by a power of two that puts the largest element in [2^13, 2^14) (exact for all that is within 2^27 of it);
// weights are 2^9 exp2(score - m) times the value's scale over the power of two above the largest that the query has seen, rounded once: 11 bits for all
// weights down to 2^-23 of the largest, and less than 2^-34 of it lost of any other.  The 2^6 left below fp16's largest number are for scores that pass m: m
// and all that was summed under it are changed only where one does so by more than 6 (as log2), or, of 32 queries, some row's maximum would
// grow in most steps of a few thousand tokens.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "anszp_cus.h"
#include "anszp_numbers.h"

namespace {

constexpr uint32_t kTileRows = 16u, kStep = 32u, kAttendWaves = 4u;      // of attend_rows_kernel
constexpr uint32_t kManyTile = 128u;                                     // rows of attend_tile_kernel's workgroup
constexpr uint32_t kMostSplits = 1024u;
constexpr float kSlack = 6.0f;                                           // (see the weights above)

struct AttendParams {
    const uint8_t* k;
    const float* k_params;
    const uint8_t* v;
    const float* v_params;
    const uint16_t* q;
    void* out;
    const int32_t* pages;
    const int32_t* lengths;
    const int32_t* starts;
    uint32_t* status;
    float* parts;                       // splits > 1: [split][tile][head][row] dimensions, unscaled sums
    float* part_stats;                  // ... and (m, l)
    uint64_t n_pages;
    uint64_t q_token_stride, q_head_stride, out_token_stride, out_head_stride;
    uint32_t n_tokens, n_seqs, n_tiles, heads, group, table_width, page_log, out_dtype;
    uint32_t splits, span;              // tokens a split covers
    uint32_t tile_rows;
    float scale;                        // times log2 e
};

// A tile of query rows: which sequence it belongs to, and what of it.
struct Tile {
    uint32_t seq, first_token, n_new, first_row, n_rows;    // n_rows 0: there is no such tile
    int32_t length;                                         // of the sequence
    bool clamped;                                           // it was given as one that the page table, or the cache, has no room for
};

__device__ __forceinline__ void flag(const AttendParams& p) {
    if (p.status) {
        atomicOr(&p.status[0], ANSZP_ST_BAD_DESC);
        atomicAdd(&p.status[1], 1u);
    }
}

// Sequences have ceil(n_new * group / rows) tiles each; every wavefront counts through them, 64 sequences at a time.
__device__ Tile find_tile(const AttendParams& p, uint32_t tile, uint32_t rows) {
    const uint32_t lane = threadIdx.x & 63u;
    Tile t = {0u, 0u, 0u, 0u, 0u, 0, false};
    uint32_t before = 0u;
    for (uint32_t s0 = 0; s0 < p.n_seqs; s0 += 64u) {
        const uint32_t s = s0 + lane;
        uint32_t a = 0u, n = 0u;
        if (s < p.n_seqs) {
            const int32_t limit = int32_t(p.n_tokens);
            const int32_t lo = min(max(p.starts[s], 0), limit), hi = min(max(p.starts[s + 1u], lo), limit);
            a = uint32_t(lo);
            n = uint32_t(hi - lo);
        }
        const uint32_t tiles = (n * p.group + rows - 1u) / rows;
        uint32_t upto = tiles;
        for (uint32_t d = 1; d < 64u; d <<= 1) {
            const uint32_t other = __shfl_up(upto, d);
            if (lane >= d) upto += other;
        }
        const uint32_t mine = tile - before - (upto - tiles);                  // wraps where the tile lies before this sequence
        const uint64_t here = __ballot(tile - before < upto && mine < tiles);
        if (here) {
            const int src = __builtin_ctzll(here);
            t.seq = s0 + uint32_t(src);
            t.first_token = __builtin_amdgcn_readlane(a, src);
            t.n_new = __builtin_amdgcn_readlane(n, src);
            t.first_row = __builtin_amdgcn_readlane(mine, src) * rows;
            t.n_rows = min(rows, t.n_new * p.group - t.first_row);
            const int64_t most = int64_t(p.table_width) << p.page_log;
            const int32_t given = p.lengths[t.seq];
            t.length = given < 0 ? 0 : given > most ? int32_t(most) : given;
            if (p.n_pages == 0u) t.length = 0;
            t.clamped = t.length != given;
            return t;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return t;
}

// positions the tile's rows see together: those below this
__device__ __forceinline__ int32_t seen_by(const AttendParams& p, const Tile& t) {
    const int32_t last_new = int32_t((t.first_row + t.n_rows - 1u) / p.group);
    return max(0, t.length - int32_t(t.n_new) + last_new + 1);
}

__device__ __forceinline__ f16x2 halves(uint32_t w) { return __builtin_bit_cast(f16x2, w); }
__device__ __forceinline__ uint32_t bits_of(f16x2 h) { return __builtin_bit_cast(uint32_t, h); }
__device__ __forceinline__ f16x2 both(float v) { return f16x2{static_cast<_Float16>(v), static_cast<_Float16>(v)}; }

// the four bytes of w less their zero-point, as fp16; offset is 1024 + z in both halves
__device__ __forceinline__ words2 less_zero(uint32_t w, f16x2 offset) {
    const uint32_t lo = __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u), hi = __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u);
    return words2{bits_of(halves(lo) - offset), bits_of(halves(hi) - offset)};
}
// ... and of bytes that are 16 times the symbols: (1024 + 16 q) / 16 - (64 + z), exact
__device__ __forceinline__ words2 less_zero_of_16(uint32_t w, f16x2 minus_64_z) {
    const uint32_t lo = __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u), hi = __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u);
    return words2{bits_of(__builtin_elementwise_fma(halves(lo), both(0.0625f), minus_64_z)), bits_of(__builtin_elementwise_fma(halves(hi), both(0.0625f), minus_64_z))};
}
// Two tokens' values of dimension e, 2^-9 of them, as fp16: the bits of a whole number q are 2^-24 q there, so that one multiplication and addition,
// q 2^-24 2^15 - z 2^-9, is exact (its inputs may be subnormal, its result is a multiple of 2^-9 below 1).  Four bits: the high halves of bytes are 16 q.
constexpr float kValueStep = 0x1p-9f;
template <uint32_t BITS>
__device__ __forceinline__ uint32_t value_pair(uint32_t first, uint32_t second, uint32_t e, f16x2 minus_zeros) {
    if constexpr (BITS == 8u) {
        return bits_of(__builtin_elementwise_fma(halves(__builtin_amdgcn_perm(second, first, 0x0C040C00u + (e & 3u) * 0x00010001u)), both(0x1p15f), minus_zeros));
    } else {
        const uint32_t bytes = __builtin_amdgcn_perm(second, first, 0x0C040C00u + ((e & 7u) >> 1) * 0x00010001u);
        return bits_of(__builtin_elementwise_fma(halves(bytes & (e & 1u ? 0x00F000F0u : 0x000F000Fu)), both(e & 1u ? 0x1p11f : 0x1p15f), minus_zeros));
    }
}
__device__ __forceinline__ f16x2 minus_zeros_of(float z0, float z1) { return f16x2{static_cast<_Float16>(z0 * -kValueStep), static_cast<_Float16>(z1 * -kValueStep)}; }

template <uint32_t BYTES>
struct Bytes {
    uint32_t w[(BYTES + 3u) / 4u];
    __device__ __forceinline__ void load(const uint8_t* p) {
        if constexpr (BYTES == 2u) {
            w[0] = *reinterpret_cast<const uint16_t*>(p);
        } else if constexpr (BYTES == 4u) {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
        } else if constexpr (BYTES == 8u) {
            const words2 t = *reinterpret_cast<const words2*>(p);
            w[0] = t[0]; w[1] = t[1];
        } else {
            for (uint32_t i = 0; i < BYTES / 16u; ++i) {
                const words4 t = reinterpret_cast<const words4*>(p)[i];
                for (uint32_t j = 0; j < 4u; ++j) w[4u * i + j] = t[j];
            }
        }
    }
};

// over the four lanes of a query: lane ^ 16, lane ^ 32
__device__ __forceinline__ float most_of_query(float v) {
    const uint32_t w = __builtin_bit_cast(uint32_t, v);
    const auto a = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    const uint32_t a0 = a[0], a1 = a[1];
    const uint32_t h = __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1)));
    const auto b = __builtin_amdgcn_permlane16_swap(h, h, false, false);
    const uint32_t b0 = b[0], b1 = b[1];
    return fmaxf(__builtin_bit_cast(float, b0), __builtin_bit_cast(float, b1));
}
// the power of two at or above a value, for values of 2^-126 .. 2^126; 0 for 0
__device__ __forceinline__ float power_above(float v) {
    return v > 0.0f ? __builtin_bit_cast(float, min((__builtin_bit_cast(uint32_t, v) + 0x7FFFFFu) & 0xFF800000u, 0x7E800000u)) : 0.0f;
}

// Few rows: 16 a workgroup, whose four wavefronts take 32 tokens each in turn.  Memory is what bounds it where it can: what a step reads
// is asked for a step ahead (two steps' worth of registers; heads of 256 leave no room for that).
// The running maximum and the values' power of two are looked up together in one vote; queries that meet a larger one rescale, the rest of the steps
// exchange nothing between lanes.  One sequence of 65000 tokens in 8 bits, 32 heads over 8, takes 27 us here, 5.2 TB/s; 48 sequences of 17 to 4100
// tokens in 4 bits, 32 heads, 113, 4.0 TB/s: with half the bytes the instructions that make operands of them, 50 % of the vector unit's time, and what a
// workgroup does before and after its tokens show.
template <uint32_t D, uint32_t BITS>
__global__ __launch_bounds__(256, 2) void attend_rows_kernel(AttendParams p) {
    constexpr uint32_t kKeyBytes = D * BITS / 32u, kValueBytes = D * BITS / 128u;      // of a key, of a value, that a lane feeds
    constexpr uint32_t kMfmas = D / 32u, kTiles = D / 16u, kVector = D * BITS / 8u;
    constexpr bool kAhead = D <= 128u;
    __shared__ float joined[kAttendWaves][kTileRows][D + 4u];
    __shared__ float stats[kAttendWaves][kTileRows][2];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15u, g = lane >> 4;
    const uint32_t head = blockIdx.y, split = blockIdx.z;
    const Tile t = find_tile(p, blockIdx.x, kTileRows);
    if (t.n_rows == 0u) return;
    if (t.clamped && t.first_row == 0u && head == 0u && split == 0u && threadIdx.x == 0u) flag(p);      // (once for a sequence)
    const int32_t seen = seen_by(p, t);
    const int32_t begin = int32_t(split * p.span), end = min(seen, begin + int32_t(p.span));
    const uint64_t part = (uint64_t(split) * p.n_tiles + blockIdx.x) * p.heads + head;
    if (p.splits > 1u && begin >= end) {                                                // nothing in this share
        if (threadIdx.x < kTileRows) reinterpret_cast<float2*>(p.part_stats)[part * kTileRows + threadIdx.x] = make_float2(-__builtin_inff(), 0.0f);
        return;
    }

    // What a step reads.  The lane feeds token c of each half as a key, tokens 4 g .. 4 g + 3 of each half as values, whose pairs (scale,
    // zero-point) it needs, like the scales of the keys of those tokens.
    struct Step {
        Bytes<kKeyBytes> keys[2];
        Bytes<kValueBytes> values[2][4];
        float key_zero[2];
        words4 key_params[2][2], value_params[2][2];
        bool there[2];
    };
    const int32_t* const table = p.pages + uint64_t(t.seq) * p.table_width;
    // Pages of 32 turns of the wavefront, a lane for each half of each: read together, so that no step waits for where it is to read.
    constexpr int32_t kTurn = int32_t(kAttendWaves * kStep);
    const int32_t own = begin + int32_t(wave * kStep);
    int32_t pages = 0;
    bool missing = false;
    const auto ask = [&](Step& s, int32_t turn) __attribute__((always_inline)) {
        const int32_t t0 = own + turn * kTurn;
        if (turn % 32 == 0) {
            const int32_t first = t0 + int32_t(lane >> 1) * kTurn + int32_t(16u * (lane & 1u));
            const int32_t read = first < end ? table[uint32_t(first) >> p.page_log] : 0;
            asm volatile("v_mov_b32 %0, %1" : "=v"(pages) : "v"(read));                 // (waited for here, not by every step that uses it)
        }
        const int32_t named[2] = {__builtin_amdgcn_readlane(pages, 2 * (turn % 32)), __builtin_amdgcn_readlane(pages, 2 * (turn % 32) + 1)};
#pragma unroll
        for (uint32_t u = 0; u < 2u; ++u) {
            const int32_t first = t0 + int32_t(16u * u);
            const bool known = named[u] >= 0 && uint64_t(named[u]) < p.n_pages;
            s.there[u] = first < end && known;
            missing |= first < end && !known;
            const uint64_t base = ((uint64_t(s.there[u] ? named[u] : 0) * p.heads + head) << p.page_log) + (uint32_t(first) & ((1u << p.page_log) - 1u) & ~15u);
            s.keys[u].load(p.k + base * kVector + (c * kVector + g * kKeyBytes));
            s.key_zero[u] = p.k_params[2u * base + (2u * c + 1u)];
            const words4* const kp = reinterpret_cast<const words4*>(p.k_params + 2u * base) + 2u * g;
            const words4* const vp = reinterpret_cast<const words4*>(p.v_params + 2u * base) + 2u * g;
            s.key_params[u][0] = kp[0]; s.key_params[u][1] = kp[1];
            s.value_params[u][0] = vp[0]; s.value_params[u][1] = vp[1];
#pragma unroll
            for (uint32_t i = 0; i < 4u; ++i) s.values[u][i].load(p.v + base * kVector + ((g * 4u + i) * kVector + c * kValueBytes));
        }
    };

    // the lane's part of query c, scaled into fp16
    const uint32_t row = t.first_row + min(c, t.n_rows - 1u), token = row / p.group, member = row - token * p.group;
    const int32_t position = t.length - int32_t(t.n_new) + int32_t(token);
    const int32_t least_position = t.length - int32_t(t.n_new) + int32_t(t.first_row / p.group);
    words4 q[kMfmas];
    float to_scores;
    {
        const uint16_t* from = p.q + uint64_t(t.first_token + token) * p.q_token_stride + uint64_t(head * p.group + member) * p.q_head_stride + g * (D / 4u);
        Eight<ANSZP_OUT_BF16> v[kMfmas];
        float most = 0.0f;
#pragma unroll
        for (uint32_t m = 0; m < kMfmas; ++m) v[m].load(from, m * 8u, 8u);
#pragma unroll
        for (uint32_t m = 0; m < kMfmas; ++m)
#pragma unroll
            for (uint32_t j = 0; j < 8u; ++j) most = fmaxf(most, fabsf(v[m][j]));
        most = most_of_query(most);
        const int32_t exponent = int32_t(__builtin_bit_cast(uint32_t, most) >> 23) - 127;
        const int32_t up = exponent == 128 ? 0 : min(13 - exponent, 126);
        const float factor = __builtin_bit_cast(float, uint32_t(up + 127) << 23);
        to_scores = p.scale * __builtin_bit_cast(float, uint32_t(127 - up) << 23);
#pragma unroll
        for (uint32_t m = 0; m < kMfmas; ++m) {
            constexpr uint32_t kOrder4[8] = {0, 2, 4, 6, 1, 3, 5, 7};                   // 4 bits: bytes of low halves, then of high ones
            f16x8 h;
#pragma unroll
            for (uint32_t j = 0; j < 8u; ++j) h[j] = static_cast<_Float16>(v[m][BITS == 4u ? kOrder4[j] : j] * factor);
            q[m] = __builtin_bit_cast(words4, h);
        }
    }

    floatx4 acc[kTiles] = {};
    float top = -__builtin_inff(), limit = top, sum = 0.0f, reach = 0.0f, less = 0.0f;  // m, what a score may reach before m is, the lane's part of l, the values' power of two and 1 over it
    const auto take = [&](const Step& step, int32_t t0) __attribute__((always_inline)) {
        float x[8], vs[8], vz[8];
#pragma unroll
        for (uint32_t u = 0; u < 2u; ++u) {
            const f16x2 offset = both(1024.0f + step.key_zero[u]), minus_64_z = both(-64.0f - step.key_zero[u]);
            floatx4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (uint32_t m = 0; m < kMfmas; ++m) {
                words2 a, b;
                if constexpr (BITS == 8u) {
                    a = less_zero(step.keys[u].w[2u * m], offset);
                    b = less_zero(step.keys[u].w[2u * m + 1u], offset);
                } else {
                    a = less_zero(step.keys[u].w[m] & 0x0F0F0F0Fu, offset);
                    b = less_zero_of_16(step.keys[u].w[m] & 0xF0F0F0F0u, minus_64_z);
                }
                s = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, words4{a[0], a[1], b[0], b[1]}), __builtin_bit_cast(f16x8, q[m]), s, 0, 0, 0);
            }
#pragma unroll
            for (uint32_t i = 0; i < 4u; ++i) {
                const uint32_t ks = step.key_params[u][i / 2u][2u * (i & 1u)], vsi = step.value_params[u][i / 2u][2u * (i & 1u)], vzi = step.value_params[u][i / 2u][2u * (i & 1u) + 1u];
                x[4u * u + i] = s[i] * (to_scores * __builtin_bit_cast(float, ks));
                vs[4u * u + i] = __builtin_bit_cast(float, vsi);
                vz[4u * u + i] = __builtin_bit_cast(float, vzi);
            }
            // (The keys' zero-points came with their scales, for other lanes' tokens.  Without a use their registers are given away while the loads are
            // still under way, and whoever gets them waits for all loads.)
            asm volatile("" ::"v"(step.key_params[u][0][1]), "v"(step.key_params[u][0][3]), "v"(step.key_params[u][1][1]), "v"(step.key_params[u][1][3]));
        }
        if (!(step.there[0] && step.there[1] && t0 + 31 <= least_position && t0 + 32 <= end)) {
            // Tokens that no row sees give nothing, whatever their numbers are; nor do, in their row, those that it does not see.
#pragma unroll
            for (uint32_t n = 0; n < 8u; ++n) {
                const int32_t place = t0 + int32_t(16u * (n / 4u) + g * 4u + n % 4u);
                const bool held = step.there[n / 4u] && place < end, sees = held && place <= position;
                x[n] = sees ? x[n] : -__builtin_inff();
                vs[n] = sees ? vs[n] : 0.0f;
                vz[n] = held ? vz[n] : 0.0f;
            }
        }
        float high = x[0], far = fabsf(vs[0]);
#pragma unroll
        for (uint32_t n = 1; n < 8u; ++n) {
            high = fmaxf(high, x[n]);
            far = fmaxf(far, fabsf(vs[n]));
        }
        if (__any(high > limit || far > reach)) {
            high = fmaxf(top, most_of_query(high));
            far = fmaxf(reach, power_above(most_of_query(far)));
            less = far > 0.0f ? 1.0f / far : 0.0f;
            const float kept = __builtin_amdgcn_exp2f(top - (high == -__builtin_inff() ? 0.0f : high)), kept_values = kept * (reach * less);
            top = high;
            limit = high + kSlack;
            reach = far;
            sum *= kept;
#pragma unroll
            for (uint32_t e = 0; e < kTiles; ++e) acc[e] *= kept_values;
        }
        const float safe = (top == -__builtin_inff() ? 0.0f : top) - (15.0f - kSlack);
        words4 weights;
#pragma unroll
        for (uint32_t n = 0; n < 8u; n += 2u) {
            const float e0 = __builtin_amdgcn_exp2f(x[n] - safe), e1 = __builtin_amdgcn_exp2f(x[n + 1u] - safe);
            sum += e0 + e1;
            weights[n / 2u] = bits_of(f16x2{static_cast<_Float16>(e0 * (vs[n] * less)), static_cast<_Float16>(e1 * (vs[n + 1u] * less))});
        }
        f16x2 z[4];
#pragma unroll
        for (uint32_t j = 0; j < 4u; ++j) z[j] = minus_zeros_of(vz[2u * j], vz[2u * j + 1u]);
#pragma unroll
        for (uint32_t e = 0; e < kTiles; ++e) {
            words4 a;
#pragma unroll
            for (uint32_t j = 0; j < 4u; ++j) {
                const Bytes<kValueBytes>&one = step.values[j >> 1][2u * (j & 1u)], &two = step.values[j >> 1][2u * (j & 1u) + 1u];
                a[j] = value_pair<BITS>(one.w[BITS == 8u ? e >> 2 : e >> 3], two.w[BITS == 8u ? e >> 2 : e >> 3], e, z[j]);
            }
            acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, weights), acc[e], 0, 0, 0);
        }
    };
    if (own < end) {
        Step one, two;
        ask(one, 0);
        // Two turns a round, the second behind the end where their number is odd: a way out between them would make the compiler wait, at the loop's
        // head, for loads that are under way on that way only.  Behind the end the first page is read, and nothing is seen.
        __builtin_amdgcn_s_waitcnt(0x0F70);                     // vmcnt(0), for the same reason
        for (int32_t turn = 0; own + turn * kTurn < end; turn += kAhead ? 2 : 1) {
            if constexpr (kAhead) {
                ask(two, turn + 1);
                __builtin_amdgcn_sched_barrier(0);
                take(one, own + turn * kTurn);
                ask(one, turn + 2);
                __builtin_amdgcn_sched_barrier(0);
                take(two, own + (turn + 1) * kTurn);
            } else {
                take(one, own + turn * kTurn);
                ask(one, turn + 1);
            }
        }
    }
    if (missing && lane == 0u) flag(p);
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);

    // the wavefronts' results together
    for (uint32_t e = 0; e < kTiles; ++e)
        for (uint32_t i = 0; i < 4u; ++i) joined[wave][c][(g * 4u + i) * kTiles + e] = acc[e][i] * (1.0f / kValueStep) * reach;
    if (g == 0u) {
        stats[wave][c][0] = top;
        stats[wave][c][1] = sum;
    }
    __syncthreads();
    const uint32_t r = threadIdx.x >> 4, d0 = (threadIdx.x & 15u) * kTiles;
    if (r >= t.n_rows) return;
    float high = -__builtin_inff(), l = 0.0f;
    for (uint32_t w = 0; w < kAttendWaves; ++w) high = fmaxf(high, stats[w][r][0]);
    const float safe = high == -__builtin_inff() ? 0.0f : high;
    float by[kAttendWaves];
    for (uint32_t w = 0; w < kAttendWaves; ++w) {
        by[w] = __builtin_amdgcn_exp2f(stats[w][r][0] - safe);
        l += stats[w][r][1] * by[w];
    }
    const float over = l == 0.0f ? 0.0f : 1.0f / l;
    const uint32_t out_row = t.first_row + r, out_token = out_row / p.group, out_member = out_row - out_token * p.group;
    const uint64_t to = uint64_t(t.first_token + out_token) * p.out_token_stride + uint64_t(head * p.group + out_member) * p.out_head_stride;
    if (p.splits > 1u && (threadIdx.x & 15u) == 0u) reinterpret_cast<float2*>(p.part_stats)[part * kTileRows + r] = make_float2(high, l);
    for (uint32_t d = 0; d < kTiles; d += 4u) {
        floatx4 o = {0.0f, 0.0f, 0.0f, 0.0f};
        for (uint32_t w = 0; w < kAttendWaves; ++w)
            for (uint32_t i = 0; i < 4u; ++i) o[i] += joined[w][r][d0 + d + i] * by[w];
        if (p.splits > 1u) {
            *reinterpret_cast<floatx4*>(p.parts + (part * kTileRows + r) * D + d0 + d) = o;
        } else if (p.out_dtype == ANSZP_OUT_BF16) {
            *reinterpret_cast<words2_any*>(static_cast<uint16_t*>(p.out) + to + d0 + d) = words2{to_bf16_pair(o[0] * over, o[1] * over), to_bf16_pair(o[2] * over, o[3] * over)};
        } else {
            *reinterpret_cast<words4_any*>(static_cast<float*>(p.out) + to + d0 + d) = __builtin_bit_cast(words4, o * over);
        }
    }
}

// 16 x n matrix of fp16 whose rows are PIECES pieces of 16 bytes: where piece j of row r lies, so that 16 lanes that read a piece of 16 consecutive
// rows meet all 64 banks (and the 16 that write 8 rows apart few of them twice).
template <uint32_t PIECES>
__host__ __device__ constexpr uint32_t place_of_piece(uint32_t r, uint32_t j) {
    if constexpr (PIECES >= 16u) return j ^ (r & 15u);
    else if constexpr (PIECES == 8u) return j ^ ((r >> 1) & 7u) ^ ((r >> 4) & 7u);
    else return j ^ ((r >> 2) & 3u) ^ ((r >> 4) & 3u);
}

// The order in which a run of COUNT loads from LDS, each for EACH matrix instructions, is issued: four loads ahead, where the compiler would have two and
// wait for every one of them.
template <uint32_t COUNT, uint32_t EACH, int RUN>
__device__ __forceinline__ void loads_ahead() {
    constexpr int kMatrix = 0x8, kFromLds = 0x100;
    __builtin_amdgcn_sched_group_barrier(kFromLds, 4, RUN);
#pragma unroll
    for (uint32_t n = 0; n < COUNT; ++n) {
        __builtin_amdgcn_sched_group_barrier(kMatrix, EACH, RUN);
        if (n + 4u < COUNT) __builtin_amdgcn_sched_group_barrier(kFromLds, 1, RUN);
    }
}

// Many rows: 128 a workgroup, 16 * RT a wavefront, T tokens a step.  Scores and weights, more than the matrix instructions, bound it, so symbols become
// operands once for all wavefronts: each thread turns some of the next step's bytes, which it asked for a step ahead, into fp16 in LDS while
// others still multiply, keys [token][dimension], values [dimension][token] with the eight tokens that a lane feeds (4 g .. 4 g + 3 of both halves of
// 32) side by side.  Otherwise as above.  Heads of 64 and 128 have four wavefronts of 32 rows, two such workgroups a CU; eight wavefronts of 32 halve
// what a row costs in staging, but all of a CU's wait for one barrier (16 sequences of 2048 tokens: 0.89 of the rate).  Heads of 256 leave room
// for 16 rows a wavefront and need the eight: two chunks of 700 tokens 78 us rather than 102 with four of 32.
// Sixteen sequences of 2048 new tokens behind up to 2048 more, 32 heads over 8 of 128, take 1740 us, 775 TFLOP/s (a large product 1330 to 1530): the
// vector unit is at work for 60 % of the time, the matrix units for 33.
template <uint32_t D, uint32_t BITS, uint32_t T, uint32_t RT, uint32_t WAVES>
__global__ __launch_bounds__(WAVES * 64u, 2) void attend_tile_kernel(AttendParams p) {
    static_assert(T == 64u, "a lane looks at one token of a step");
    constexpr uint32_t kThreads = WAVES * 64u;
    constexpr uint32_t kMfmas = D / 32u, kTiles = D / 16u, kVector = D * BITS / 8u, kRows = 16u * WAVES * RT;
    constexpr uint32_t kKeyDims = T * D / kThreads, kValueDims = T * D / (4u * kThreads);             // a thread's: of one key; of each of four values
    constexpr uint32_t kKeyBytes = kKeyDims * BITS / 8u, kValueBytes = kValueDims * BITS / 8u, kChunks = D / kValueDims;
    constexpr uint32_t kKeyPieces = D / 8u, kValuePieces = T / 8u;
    __shared__ words4 key_buffer[2][T][kKeyPieces];
    __shared__ words2 value_buffer[2][D][kValuePieces * 2u];
    alignas(16) __shared__ float key_scales[2][T], value_scales[2][T], ratios[WAVES][T];            // (a wavefront's own: value scales over its power of two)
    __shared__ uint32_t known[2][T / 16u];
    __shared__ int32_t lost[2];                                                         // the last step whose buffer lacks pages
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15u, g = lane >> 4;
    const uint32_t head = blockIdx.x % p.heads, tile = p.n_tiles - 1u - blockIdx.x / p.heads;       // (later tokens see more: first)
    const uint32_t split = blockIdx.y;
    const Tile t = find_tile(p, tile, kRows);
    if (t.n_rows == 0u) return;
    if (t.clamped && t.first_row == 0u && head == 0u && split == 0u && threadIdx.x == 0u) flag(p);
    const int32_t begin = int32_t(split * p.span), end = min(seen_by(p, t), begin + int32_t(p.span));
    const uint64_t part = (uint64_t(split) * p.n_tiles + tile) * p.heads + head;
    if (p.splits > 1u && begin >= end) {
        if (threadIdx.x < kRows) reinterpret_cast<float2*>(p.part_stats)[part * kRows + threadIdx.x] = make_float2(-__builtin_inff(), 0.0f);
        return;
    }

    // staging
    const uint32_t key_token = threadIdx.x / (kThreads / T), key_part = threadIdx.x % (kThreads / T);
    const uint32_t quad = threadIdx.x / kChunks, chunk = threadIdx.x % kChunks;
    const int32_t* const table = p.pages + uint64_t(t.seq) * p.table_width;
    const auto page_at = [&](int32_t place) __attribute__((always_inline)) { return table[place < end ? uint32_t(place) >> p.page_log : 0u]; };
    bool missing = false;
    if (threadIdx.x < 2u) lost[threadIdx.x] = -1;
    Bytes<kKeyBytes> key_bytes;
    Bytes<kValueBytes> value_bytes[4];
    float2 key_pair;
    float value_scale;                                                                  // of the key's token
    words4 value_pairs[2];
    int32_t key_page, value_page;                                                       // of the step to be asked for next
    bool key_there, value_there;                                                        // of what has been asked for
    const auto ask_pages = [&](int32_t step) __attribute__((always_inline)) {
        key_page = page_at(begin + step * int32_t(T) + int32_t(key_token));
        value_page = page_at(begin + step * int32_t(T) + int32_t(quad * 4u));
    };
    const auto vector_at = [&](int32_t place, int32_t page, bool there) __attribute__((always_inline)) {     // (a cache has fewer than 2^32)
        return ((uint32_t(there ? page : 0) * p.heads + head) << p.page_log) + (uint32_t(place) & ((1u << p.page_log) - 1u));
    };
    const auto ask = [&](int32_t step) __attribute__((always_inline)) {
        const int32_t key_place = begin + step * int32_t(T) + int32_t(key_token), value_place = begin + step * int32_t(T) + int32_t(quad * 4u);
        const bool key_known = uint32_t(key_page) < uint32_t(p.n_pages), value_known = uint32_t(value_page) < uint32_t(p.n_pages);
        missing |= key_place < end && !key_known;
        key_there = key_place < end && key_known;
        value_there = value_place < end && value_known;
        const uint32_t kv = vector_at(key_place, key_page, key_there), vv = vector_at(value_place, value_page, value_there);
        key_bytes.load(p.k + uint64_t(kv) * kVector + key_part * kKeyBytes);
        key_pair = reinterpret_cast<const float2*>(p.k_params)[kv];
        value_scale = p.v_params[2u * uint64_t(kv)];
#pragma unroll
        for (uint32_t i = 0; i < 4u; ++i) value_bytes[i].load(p.v + uint64_t(vv) * kVector + (i * kVector + chunk * kValueBytes));
        value_pairs[0] = reinterpret_cast<const words4*>(p.v_params)[vv / 2u];
        value_pairs[1] = reinterpret_cast<const words4*>(p.v_params)[vv / 2u + 1u];
    };
    const auto put = [&](int32_t step) __attribute__((always_inline)) {
        const uint32_t to = uint32_t(step) & 1u;
        const float key_zero = key_there ? key_pair.y : 0.0f;
        const f16x2 offset = both(1024.0f + key_zero), minus_64_z = both(-64.0f - key_zero);
#pragma unroll
        for (uint32_t j = 0; j < kKeyDims / 8u; ++j) {
            words2 a, b;
            if constexpr (BITS == 8u) {
                a = less_zero(key_bytes.w[2u * j], offset);
                b = less_zero(key_bytes.w[2u * j + 1u], offset);
            } else {
                a = less_zero(key_bytes.w[j] & 0x0F0F0F0Fu, offset);
                b = less_zero_of_16(key_bytes.w[j] & 0xF0F0F0F0u, minus_64_z);
            }
            key_buffer[to][key_token][place_of_piece<kKeyPieces>(key_token, key_part * (kKeyDims / 8u) + j)] = words4{a[0], a[1], b[0], b[1]};
        }
        if (key_part == 0u) {
            // A value without a scale makes its key's NaN: rows that see the token get NaN, and the weights of others stay 0.
            const bool held = key_there && begin + step * int32_t(T) + int32_t(key_token) < end, sound = fabsf(value_scale) < __builtin_inff();
            key_scales[to][key_token] = sound ? key_pair.x : __builtin_nanf("");
            value_scales[to][key_token] = held && sound ? value_scale : 0.0f;
        }
        float vz[4];
#pragma unroll
        for (uint32_t i = 0; i < 4u; ++i) {
            const uint32_t zi = value_pairs[i / 2u][2u * (i & 1u) + 1u];
            asm volatile("" ::"v"(value_pairs[i / 2u][2u * (i & 1u)]));                 // (the scale came with it: see attend_rows_kernel)
            vz[i] = __builtin_bit_cast(float, zi);
        }
        if (!value_there || begin + (step + 1) * int32_t(T) > end) {                    // what lies behind the end, and pages that are not there
#pragma unroll
            for (uint32_t i = 0; i < 4u; ++i) {
                vz[i] = value_there && begin + step * int32_t(T) + int32_t(quad * 4u + i) < end ? vz[i] : 0.0f;
            }
        }
        const f16x2 z0 = minus_zeros_of(vz[0], vz[1]), z1 = minus_zeros_of(vz[2], vz[3]);
        // the quad's place among the 32 tokens of its group: half (quad / 4) % 2 of piece quad % 4
        const uint32_t piece = quad / 8u * 4u + (quad & 3u), half = (quad >> 2) & 1u;
#pragma unroll
        for (uint32_t e = 0; e < kValueDims; ++e) {
            const uint32_t w = BITS == 8u ? e >> 2 : e >> 3;
            const uint32_t dim = chunk * kValueDims + e;
            value_buffer[to][dim][2u * place_of_piece<kValuePieces>(dim, piece) + half] =
                words2{value_pair<BITS>(value_bytes[0].w[w], value_bytes[1].w[w], e, z0), value_pair<BITS>(value_bytes[2].w[w], value_bytes[3].w[w], e, z1)};
        }
        if (key_part == 0u && (key_token & 15u) == 0u) {
            known[to][key_token / 16u] = key_there ? 1u : 0u;
            if (!key_there && begin + step * int32_t(T) + int32_t(key_token) < end) lost[to] = step;
        }
    };

    // the wavefront's queries, scaled into fp16
    const uint32_t own_row = t.first_row + wave * (16u * RT), last_row = t.first_row + t.n_rows - 1u;
    words4 q[RT][kMfmas];
    float to_exponent[RT];
    int32_t position[RT];
#pragma unroll
    for (uint32_t b = 0; b < RT; ++b) {
        const uint32_t row = min(own_row + 16u * b + c, last_row), token = row / p.group, member = row - token * p.group;
        position[b] = t.length - int32_t(t.n_new) + int32_t(token);
        const uint16_t* from = p.q + uint64_t(t.first_token + token) * p.q_token_stride + uint64_t(head * p.group + member) * p.q_head_stride + g * 8u;
        Eight<ANSZP_OUT_BF16> v[kMfmas];
        float most = 0.0f;
#pragma unroll
        for (uint32_t m = 0; m < kMfmas; ++m) v[m].load(from, m * 32u, 8u);
#pragma unroll
        for (uint32_t m = 0; m < kMfmas; ++m)
#pragma unroll
            for (uint32_t j = 0; j < 8u; ++j) most = fmaxf(most, fabsf(v[m][j]));
        most = most_of_query(most);
        const int32_t exponent = int32_t(__builtin_bit_cast(uint32_t, most) >> 23) - 127;
        const int32_t up = exponent == 128 ? 0 : min(13 - exponent, 126);
        // Scores are kept without the factor that makes them exponents, which is positive: the scale's sign (and a scale of 0) go with the queries.
        const float factor = __builtin_bit_cast(float, uint32_t(up + 127) << 23) * (p.scale > 0.0f ? 1.0f : p.scale < 0.0f ? -1.0f : 0.0f * p.scale);
        to_exponent[b] = fmaxf(fabsf(p.scale) * __builtin_bit_cast(float, uint32_t(127 - up) << 23), 0x1p-126f);
#pragma unroll
        for (uint32_t m = 0; m < kMfmas; ++m) {
            constexpr uint32_t kOrder4[8] = {0, 2, 4, 6, 1, 3, 5, 7};
            f16x8 h;
#pragma unroll
            for (uint32_t j = 0; j < 8u; ++j) h[j] = static_cast<_Float16>(v[m][BITS == 4u ? kOrder4[j] : j] * factor);
            q[b][m] = __builtin_bit_cast(words4, h);
        }
    }
    const int32_t least_position = t.length - int32_t(t.n_new) + int32_t(min(own_row, last_row) / p.group);
    const int32_t most_position = own_row > last_row ? -1 : t.length - int32_t(t.n_new) + int32_t(min(own_row + 16u * RT - 1u, last_row) / p.group);

    floatx4 acc[kTiles][RT] = {}, sum[RT] = {};                                        // (sums: products with ones, alike in all four)
    const uint32_t one = 0x3C003C00u;
    // m, 1 over the power of two above the value scales that the row has seen (0: none); the least of those powers among rows that still see any
    float top[RT], less[RT], settled = 0.0f;
    const auto reach_of = [](float one_over) __attribute__((always_inline)) { return one_over > 0.0f ? 1.0f / one_over : 0.0f; };
#pragma unroll
    for (uint32_t b = 0; b < RT; ++b) {
        top[b] = -__builtin_inff();
        less[b] = 0.0f;
    }
    // Places are exclusive ors of what r and j give, so that the lane's own part, of row c and piece g, and the rest of a row and piece make up any of them: one
    // register for all addresses, and registers are what loads from LDS can be under way in.
    const uint32_t key_own = 16u * (c * kKeyPieces + place_of_piece<kKeyPieces>(c, g)), value_own = 16u * (c * kValuePieces + place_of_piece<kValuePieces>(c, g));
    // APART: the tile's rows do not all see all of the step's tokens, and each has its own power of two from here on; before, all have the same.
    const auto take = [&](int32_t step, auto apart) __attribute__((always_inline)) {
        constexpr bool kApart = decltype(apart)::value;
        if (most_position < 0) return;                                                  // (no rows, or none that see anything)
        const uint32_t in = uint32_t(step) & 1u;
        const uint32_t key_at = key_own + in * uint32_t(sizeof key_buffer[0]), value_at = value_own + in * uint32_t(sizeof value_buffer[0]);
        const float scale = value_scales[in][lane];
        const bool larger = __any(fabsf(scale) > settled);
        float rescaled[RT];
#pragma unroll
        for (uint32_t b = 0; b < RT; ++b) rescaled[b] = 1.0f;
        if (larger) {                                                                   // values larger than any that some row has seen
            float upto = fabsf(scale);                                                  // the largest of the step's tokens up to the lane's own
            for (uint32_t d = 1; d < 64u; d <<= 1) {
                const float other = __shfl_up(upto, d);
                if (lane >= d) upto = fmaxf(upto, other);
            }
            float lowest = __builtin_inff();
#pragma unroll
            for (uint32_t b = 0; b < RT; ++b) {
                const int32_t last = min(position[b] - (begin + step * int32_t(T)), 63);          // of the step's tokens, that the row sees
                const float seen = __shfl(upto, max(last, 0)), before = reach_of(less[b]);
                const float now = last < 0 ? before : fmaxf(before, power_above(seen));
                if (last >= 0) lowest = fminf(lowest, now);                             // (the others see nothing any more)
                less[b] = now > 0.0f ? 1.0f / now : 0.0f;
                rescaled[b] = before * less[b];                                         // (done with the maximum's, below)
            }
            for (int x = 8; x; x >>= 1) lowest = fminf(lowest, __shfl_xor(lowest, x));
            settled = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int32_t, lowest)));
        }
        if constexpr (!kApart) ratios[wave][lane] = scale * less[0];
        const bool lacking = lost[in] == step;
#pragma unroll
        for (uint32_t h = 0; h < T / 32u; ++h) {
            const int32_t t0 = begin + step * int32_t(T) + int32_t(32u * h);
            if (kApart && (t0 > most_position || t0 >= end)) break;                     // nothing that these rows see
            float y[RT][8];
#pragma unroll
            for (uint32_t u = 0; u < 2u; ++u) {
                const uint32_t row = 32u * h + 16u * u;
                floatx4 s[RT] = {};
#pragma unroll
                for (uint32_t m = 0; m < kMfmas; ++m) {
                    const uint32_t at = (key_at ^ 16u * place_of_piece<kKeyPieces>(row, m * 4u)) + 16u * row * kKeyPieces;
                    const words4 a = *reinterpret_cast<const words4*>(reinterpret_cast<const uint8_t*>(key_buffer) + at);
#pragma unroll
                    for (uint32_t b = 0; b < RT; ++b) s[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, q[b][m]), s[b], 0, 0, 0);
                }
                const floatx4 ks = *reinterpret_cast<const floatx4*>(&key_scales[in][32u * h + 16u * u + 4u * g]);
#pragma unroll
                for (uint32_t b = 0; b < RT; ++b)
#pragma unroll
                    for (uint32_t i = 0; i < 4u; ++i) y[b][4u * u + i] = s[b][i] * ks[i];
            }
            loads_ahead<2u * kMfmas, RT, 1>();
            const bool whole = !lacking && (!kApart || t0 + 31 <= least_position) && t0 + 32 <= end;
            if (!whole) {
#pragma unroll
                for (uint32_t n = 0; n < 8u; ++n) {
                    const int32_t place = t0 + int32_t(16u * (n / 4u) + g * 4u + n % 4u);
                    const bool held = place < end && known[in][2u * h + n / 4u];
#pragma unroll
                    for (uint32_t b = 0; b < RT; ++b)
                        y[b][n] = held && (!kApart || place <= position[b]) ? y[b][n] : -__builtin_inff();
                }
            }
            bool grows = false;
            float high[RT];
#pragma unroll
            for (uint32_t b = 0; b < RT; ++b) {
                high[b] = fmaxf(y[b][0], y[b][1]);
#pragma unroll
                for (uint32_t n = 2; n < 8u; n += 2u) high[b] = fmaxf(fmaxf(high[b], y[b][n]), y[b][n + 1u]);
                grows |= (high[b] - top[b]) * to_exponent[b] > kSlack;
            }
            const bool moves = __any(grows);
            if (moves || (h == 0u && larger)) {
#pragma unroll
                for (uint32_t b = 0; b < RT; ++b) {
                    const float now = moves ? fmaxf(top[b], most_of_query(high[b])) : top[b];
                    const float kept = moves ? __builtin_amdgcn_exp2f((top[b] - (now == -__builtin_inff() ? 0.0f : now)) * to_exponent[b]) : 1.0f;
                    const float kept_values = h == 0u ? kept * rescaled[b] : kept;
                    top[b] = now;
                    sum[b] *= kept;
#pragma unroll
                    for (uint32_t e = 0; e < kTiles; ++e) acc[e][b] *= kept_values;
                }
            }
            const float* const scales = kApart ? &value_scales[in][32u * h + 4u * g] : &ratios[wave][32u * h + 4u * g];
            const floatx4 vs[2] = {reinterpret_cast<const floatx4*>(scales)[0], reinterpret_cast<const floatx4*>(scales)[4]};
            words4 weights[RT];
#pragma unroll
            for (uint32_t b = 0; b < RT; ++b) {
                words4 plain;
                const float less_top = 15.0f - kSlack - (top[b] == -__builtin_inff() ? 0.0f : top[b]) * to_exponent[b];
#pragma unroll
                for (uint32_t n = 0; n < 8u; n += 2u) {
                    const float e0 = __builtin_amdgcn_exp2f(fmaf(y[b][n], to_exponent[b], less_top)), e1 = __builtin_amdgcn_exp2f(fmaf(y[b][n + 1u], to_exponent[b], less_top));
                    plain[n / 2u] = bits_of(f16x2{static_cast<_Float16>(e0), static_cast<_Float16>(e1)});
                    // Rounded once.  (In this order nothing is left of a token that the row does not see, however far it is above the row's power of two.)
                    const float by = kApart ? less[b] : 1.0f;
                    weights[b][n / 2u] = bits_of(f16x2{static_cast<_Float16>(e0 * vs[n / 4u][n & 3u] * by), static_cast<_Float16>(e1 * vs[n / 4u][(n + 1u) & 3u] * by)});
                }
                sum[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, words4{one, one, one, one}), __builtin_bit_cast(f16x8, plain), sum[b], 0, 0, 0);
            }
#pragma unroll
            for (uint32_t e = 0; e < kTiles; ++e) {
                const uint32_t at = (value_at ^ 16u * place_of_piece<kValuePieces>(16u * e, 4u * h)) + 256u * e * kValuePieces;
                const words4 a = *reinterpret_cast<const words4*>(reinterpret_cast<const uint8_t*>(value_buffer) + at);
#pragma unroll
                for (uint32_t b = 0; b < RT; ++b) acc[e][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, weights[b]), acc[e][b], 0, 0, 0);
            }
            loads_ahead<kTiles, RT, 0>();
        }
    };
    const int32_t steps = (max(0, end - begin) + int32_t(T) - 1) / int32_t(T);
    if (steps > 0) {
        ask_pages(0);
        ask(0);
        ask_pages(1);
        __syncthreads();                                                                // (`lost` is cleared)
        put(0);
        ask(1);
        ask_pages(2);
        __syncthreads();
        // Steps that all of the tile's rows see whole first: they have less to look at.
        const int32_t shared = max(0, t.length - int32_t(t.n_new) + int32_t(t.first_row / p.group) + 1 - begin) / int32_t(T);
        const auto round = [&](int32_t step, auto apart) __attribute__((always_inline)) {
            take(step, apart);
            put(step + 1);                                                              // (behind the end: nothing that is looked at)
            ask(step + 2);
            ask_pages(step + 3);
            __syncthreads();
        };
        int32_t step = 0;
        for (; step < min(shared, steps); ++step) round(step, std::false_type{});
        for (; step < steps; ++step) round(step, std::true_type{});
    }
    if (missing) flag(p);
#pragma unroll
    for (uint32_t b = 0; b < RT; ++b) {
        const float l = sum[b][0];
        const uint32_t r = wave * (16u * RT) + 16u * b + c;
        if (r >= t.n_rows) continue;
        const uint32_t row = t.first_row + r, token = row / p.group, member = row - token * p.group;
        const uint64_t out_at = uint64_t(t.first_token + token) * p.out_token_stride + uint64_t(head * p.group + member) * p.out_head_stride;
        const float over = p.splits > 1u ? reach_of(less[b]) : l == 0.0f ? 0.0f : reach_of(less[b]) / l;
        if (p.splits > 1u && g == 0u) reinterpret_cast<float2*>(p.part_stats)[part * kRows + r] = make_float2(top[b] * to_exponent[b], l);
#pragma unroll
        for (uint32_t e = 0; e < kTiles; ++e) {
            const floatx4 o = acc[e][b] * (1.0f / kValueStep) * over;
            const uint32_t d = 16u * e + 4u * g;
            if (p.splits > 1u)
                *reinterpret_cast<floatx4*>(p.parts + (part * kRows + r) * D + d) = o;
            else if (p.out_dtype == ANSZP_OUT_BF16)
                *reinterpret_cast<words2_any*>(static_cast<uint16_t*>(p.out) + out_at + d) = words2{to_bf16_pair(o[0], o[1]), to_bf16_pair(o[2], o[3])};
            else
                *reinterpret_cast<words4_any*>(static_cast<float*>(p.out) + out_at + d) = __builtin_bit_cast(words4, o);
        }
    }
}

// The splits' results together: a workgroup for every fourth row of a tile and head, if it has as many, a row at a time; D / 4 lanes have a split, their sums meet in LDS.  32 rows of 64
// splits each take 5 us, most of it a launch.
template <uint32_t D>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendParams p) {
    constexpr uint32_t kLanes = D / 4u, kGroups = 256u / kLanes;
    __shared__ floatx4 joined[kGroups][kLanes];
    __shared__ float sums[kGroups], tops[4];
    __shared__ float2 stats_of[kMostSplits];
    const uint32_t head = blockIdx.y;
    const Tile t = find_tile(p, blockIdx.x, p.tile_rows);
    const uint32_t d = threadIdx.x % kLanes, n = threadIdx.x / kLanes;
    const float2* stats = reinterpret_cast<const float2*>(p.part_stats);
    for (uint32_t r = blockIdx.z; r < t.n_rows; r += gridDim.z) {
        const auto part_of = [&](uint32_t s) { return ((uint64_t(s) * p.n_tiles + blockIdx.x) * p.heads + head) * p.tile_rows + r; };
        float high = -__builtin_inff();
        for (uint32_t s = threadIdx.x; s < p.splits; s += 256u) {
            stats_of[s] = stats[part_of(s)];
            high = fmaxf(high, stats_of[s].x);
        }
        for (int x = 32; x; x >>= 1) high = fmaxf(high, __shfl_xor(high, x));
        if ((threadIdx.x & 63u) == 0u) tops[threadIdx.x >> 6] = high;
        __syncthreads();
        high = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
        const float safe = high == -__builtin_inff() ? 0.0f : high;
        floatx4 o = {0.0f, 0.0f, 0.0f, 0.0f};
        float l = 0.0f;
        for (uint32_t first = n; first < p.splits; first += 4u * kGroups) {               // four of them under way
            floatx4 part[4];
#pragma unroll
            for (uint32_t u = 0; u < 4u; ++u)
                part[u] = *reinterpret_cast<const floatx4*>(p.parts + part_of(min(first + u * kGroups, p.splits - 1u)) * D + 4u * d);
#pragma unroll
            for (uint32_t u = 0; u < 4u; ++u) {
                const uint32_t s = first + u * kGroups;
                const float2 w = stats_of[min(s, p.splits - 1u)];
                if (s >= p.splits || w.y == 0.0f) continue;                                 // (where the sum is nothing no part was written)
                const float by = __builtin_amdgcn_exp2f(w.x - safe);
                l += w.y * by;
                o += part[u] * by;
            }
        }
        joined[n][d] = o;
        if (d == 0u) sums[n] = l;
        __syncthreads();
        if (n == 0u) {
            for (uint32_t m = 1; m < kGroups; ++m) {
                o += joined[m][d];
                l += sums[m];
            }
            const float over = l == 0.0f ? 0.0f : 1.0f / l;
            const uint32_t row = t.first_row + r, token = row / p.group, member = row - token * p.group;
            const uint64_t to = uint64_t(t.first_token + token) * p.out_token_stride + uint64_t(head * p.group + member) * p.out_head_stride + 4u * d;
            o *= over;
            if (p.out_dtype == ANSZP_OUT_BF16)
                *reinterpret_cast<words2_any*>(static_cast<uint16_t*>(p.out) + to) = words2{to_bf16_pair(o[0], o[1]), to_bf16_pair(o[2], o[3])};
            else
                *reinterpret_cast<words4_any*>(static_cast<float*>(p.out) + to) = __builtin_bit_cast(words4, o);
        }
        __syncthreads();
    }
}

// Above so many rows per sequence and head of the cache, on average, attend_tile_kernel is the faster one: it reads tokens once for 128 rows, not 16, but
// vectors of few bytes are no work for attend_rows_kernel.  16 sequences of 2000 to 4000 tokens, 8 heads, few rows' kernel and many rows', us:
//   128 x 8 bits: 16 rows 42 and 61, 32 rows 58 and 63, 48 rows 69 and 67, 128 rows 131 and 100
//   256 x 8 bits: 16 rows 61 and 85, 32 rows 89 and 89, 48 rows 107 and 93
//   64 x 8 bits:  32 rows 37 and 52, 64 rows 50 and 68, 128 rows 81 and 81
//   128 x 4 bits: 32 rows 44 and 64, 64 rows 60 and 85, 128 rows 97 and 97
// (An average: single tokens beside a chunk take the chunk's kernel.  32 of them behind 18500 to 65000 tokens, 8 heads of four queries, take 578 us, a chunk of 1531
// 92, both in one call 1974.)
uint64_t few_rows_of(const anszp_cache_t& c) { return c.head_dim * c.bits / 8u <= 64u ? 96u : 32u; }

// How the tokens are shared out: enough workgroups to fill the chip, of at least 256 tokens each; and where there are more than that, shares of a
// length, since sequences differ in theirs and the longest would end last.  A share costs its workgroup's start and its part of the join, so many workgroups
// have longer ones (us, with a share for 1408 and for 2816 tokens):
//   48 sequences of 17 to 4100 tokens, 32 heads in 4 bits 123 and 120 (123 with one workgroup for all of a sequence's tokens), in 8 bits 180 and 180 (190 with one);
//   200 of 10 to 2000, 8 heads in 4 bits 73.5 and 62.7;    64 of 100 to 4000, 8 heads of four queries in 8 bits 69 and 76;    16, 32 heads in 4 bits 44 and 46.6.
// The lengths are on the device: what the page tables can hold counts, and a table wider than its sequences makes longer shares (8 heads of four queries, a table
// for 4000 tokens and one for 65500: one sequence of 4000 tokens 11 and 16.5 us, four 20 and 22, 64 of 100 to 4000 69 and 82).
struct Shares {
    uint32_t rows, tiles, splits, span;     // rows of a tile: attend_rows_kernel's, or attend_tile_kernel's
};
Shares shares_of(const anszp_attend_args_t& a) {
    Shares s;
    const bool many = a.n_tokens * a.group > few_rows_of(a.cache) * a.n_seqs;
    s.rows = many ? kManyTile : kTileRows;
    s.tiles = static_cast<uint32_t>(a.n_tokens * a.group / s.rows + a.n_seqs);
    const uint64_t most = uint64_t(a.table_width) * a.cache.page_size, groups = std::max<uint64_t>(1u, uint64_t(s.tiles) * a.cache.heads), cus = device_cus();
    uint64_t splits = 2u * cus / groups;
    const uint64_t share = groups < 4u * cus ? 1408u : 2816u;
    if (!many) splits = std::max(splits, std::min<uint64_t>(32u * cus / groups, (most + share - 1u) / share));
    splits = std::max<uint64_t>(1u, std::min<uint64_t>(std::min<uint64_t>(splits, (most + 255u) / 256u), kMostSplits));
    const uint64_t whole = 2u * kStep * kAttendWaves;                                   // (the few rows' wavefronts take two turns a round)
    s.span = static_cast<uint32_t>((most + splits * whole - 1u) / (splits * whole) * whole);
    s.splits = static_cast<uint32_t>((most + s.span - 1u) / s.span);
    return s;
}

bool in_range(const anszp_attend_args_t& a) {
    const anszp_cache_t& c = a.cache;
    return !(a.n_tokens >= 1u << 24 || a.n_seqs >= 1u << 24 || a.table_width == 0u || uint64_t(a.table_width) * c.page_size > 1ull << 30 || a.group == 0u ||
             a.group > 256u || (a.out_dtype != ANSZP_OUT_F32 && a.out_dtype != ANSZP_OUT_BF16) || (a.n_tokens * a.group / kTileRows + a.n_seqs) * c.heads >= 1ull << 31);
}

// A launch leaves out what is beyond 2^32 threads in a dimension, without an error.
bool fits_a_launch(const anszp_attend_args_t& a, const Shares& s) {
    const uint64_t groups = s.rows == kTileRows ? s.tiles : uint64_t(s.tiles) * a.cache.heads;
    return groups * (s.rows == kTileRows || a.cache.head_dim < 256u ? 256u : 512u) < 1ull << 32 && uint64_t(s.tiles) * 256u < 1ull << 32;
}

uint64_t workspace_of(const anszp_attend_args_t& a, const Shares& s) {
    return s.splits > 1u ? uint64_t(s.splits) * s.tiles * a.cache.heads * s.rows * (a.cache.head_dim + 2u) * sizeof(float) : 0u;
}

template <uint32_t D>
void launch(const AttendParams& p, uint32_t bits, hipStream_t s) {
    if (p.tile_rows == kTileRows) {
        const dim3 grid(p.n_tiles, p.heads, p.splits);
        if (bits == 8u) hipLaunchKernelGGL((attend_rows_kernel<D, 8u>), grid, dim3(256), 0, s, p);
        else hipLaunchKernelGGL((attend_rows_kernel<D, 4u>), grid, dim3(256), 0, s, p);
    } else {
        constexpr uint32_t RT = D == 256u ? 1u : 2u, WAVES = kManyTile / (16u * RT);
        const dim3 grid(p.n_tiles * p.heads, p.splits);
        if (bits == 8u) hipLaunchKernelGGL((attend_tile_kernel<D, 8u, 64u, RT, WAVES>), grid, dim3(WAVES * 64u), 0, s, p);
        else hipLaunchKernelGGL((attend_tile_kernel<D, 4u, 64u, RT, WAVES>), grid, dim3(WAVES * 64u), 0, s, p);
    }
    if (p.splits > 1u) {
        const uint64_t rows = (uint64_t(p.n_tokens) * p.group + p.n_seqs - 1u) / p.n_seqs;         // of a sequence and head
        hipLaunchKernelGGL(attend_join_kernel<D>, dim3(p.n_tiles, p.heads, static_cast<uint32_t>(std::min<uint64_t>(p.tile_rows / 4u, rows))), dim3(256), 0, s, p);
    }
}

}  // namespace

extern "C" {

uint64_t anszp_attend_workspace_bytes(const anszp_attend_args_t* a) {
    if (!a || !in_range(*a) || a->n_tokens == 0u || a->n_seqs == 0u) return 0u;
    return workspace_of(*a, shares_of(*a));
}

int anszp_attend(const anszp_attend_args_t* a, void* hip_stream) {
    if (!a) return ANSZP_E_NULL;
    const int rc = anszp_cache_check(&a->cache);
    if (rc) return rc;
    if (!in_range(*a)) return ANSZP_E_RANGE;
    if (a->n_tokens == 0u || a->n_seqs == 0u) return ANSZP_OK;
    if (!a->q || !a->out || !a->pages || !a->lengths || !a->starts) return ANSZP_E_NULL;
    if ((a->n_tokens > 1u && a->out_token_stride < a->cache.head_dim) || (a->cache.heads * a->group > 1u && a->out_head_stride < a->cache.head_dim)) return ANSZP_E_RANGE;
    const Shares s = shares_of(*a);
    if (!fits_a_launch(*a, s)) return ANSZP_E_RANGE;
    const uint64_t need = workspace_of(*a, s);
    if (need && !a->workspace) return ANSZP_E_NULL;
    if (a->workspace_bytes < need || (reinterpret_cast<uintptr_t>(a->workspace) & 15u)) return ANSZP_E_RANGE;
    AttendParams p = {};
    p.k = a->cache.k; p.k_params = a->cache.k_params; p.v = a->cache.v; p.v_params = a->cache.v_params;
    p.q = static_cast<const uint16_t*>(a->q); p.out = a->out; p.pages = a->pages; p.lengths = a->lengths; p.starts = a->starts; p.status = a->status;
    p.parts = static_cast<float*>(a->workspace);
    p.part_stats = p.parts + uint64_t(s.splits) * s.tiles * a->cache.heads * s.rows * a->cache.head_dim;
    p.tile_rows = s.rows;
    p.n_pages = a->cache.n_pages;
    p.q_token_stride = a->q_token_stride; p.q_head_stride = a->q_head_stride; p.out_token_stride = a->out_token_stride; p.out_head_stride = a->out_head_stride;
    p.n_tokens = static_cast<uint32_t>(a->n_tokens); p.n_seqs = static_cast<uint32_t>(a->n_seqs); p.n_tiles = s.tiles;
    p.heads = a->cache.heads; p.group = a->group; p.table_width = a->table_width; p.page_log = static_cast<uint32_t>(__builtin_ctz(a->cache.page_size));
    p.out_dtype = a->out_dtype; p.splits = s.splits; p.span = s.span;
    p.scale = a->scale * 1.4426950408889634f;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (a->cache.head_dim == 64u) launch<64u>(p, a->cache.bits, stream);
    else if (a->cache.head_dim == 128u) launch<128u>(p, a->cache.bits, stream);
    else launch<256u>(p, a->cache.bits, stream);
    return hipGetLastError() == hipSuccess ? ANSZP_OK : ANSZP_E_HIP;
}

}  // extern "C"
