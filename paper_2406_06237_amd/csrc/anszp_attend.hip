// Attention of new tokens over the quantised paged cache, for gfx950:
//   out = sum_t softmax_t(scale * q . k_t) v_t,      k_t = s_t (symbol - z_t),  v_t alike.
// One pass over the tokens with the running maximum m and sum l of each query's weights, 32 tokens a step, products in
// v_mfma_f32_16x16x32_f16.  The rows of a tile are the queries of one head of the cache: (new token, query head of the group).
//
// Symbols become matrix operands in registers.  fp16 holds 1024 + q for every byte q as the bits 0x6400 | q, so symbol - z is
// one bitwise step and one packed subtraction of 1024 + z, exact.  A key's scale multiplies its scores; a value's scale goes into the weight.
//   scores^T = K Q^T: lane (c, g), c = lane % 16, g = lane / 16, feeds a key's dimensions [g D / 4, (g + 1) D / 4), which lie one behind
//     the other in memory, and ends up with the scores of query c for tokens 4 g .. 4 g + 3 of each half of the step;
//   out^T = V^T P^T: those are the weights the lane has to feed for query c, so they never leave their lane.  It feeds, for the same tokens,
//     the dimensions [c D / 16, (c + 1) D / 16) of their values, 16 lanes reading a value end to end, and the bytes of one dimension
//     are brought together by v_perm_b32.  Nothing passes through LDS but the join of the wavefronts' results.
// Queries are scaled per row by a power of two that puts the largest element in [2^13, 2^14) (exact for all that is within 2^27 of it);
// weights are 2^15 exp2(score - m) times the value's scale over the power of two above the largest seen: 11 bits for all weights down
// to 2^-29 of the largest.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "anszp_cus.h"
#include "anszp_numbers.h"

namespace {

constexpr uint32_t kTileRows = 16u, kStep = 32u, kAttendWaves = 4u;

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
    float scale;                        // times log2 e
};

// A tile of query rows: which sequence it belongs to, and what of it.
struct Tile {
    uint32_t seq, first_token, n_new, first_row, n_rows;    // n_rows 0: there is no such tile
    int32_t length;                                         // of the sequence
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
    Tile t = {0u, 0u, 0u, 0u, 0u, 0};
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
            t.first_token = __shfl(a, src);
            t.n_new = __shfl(n, src);
            t.first_row = __shfl(mine, src) * rows;
            t.n_rows = min(rows, t.n_new * p.group - t.first_row);
            const int64_t most = int64_t(p.table_width) << p.page_log;
            const int32_t given = p.lengths[t.seq];
            t.length = given < 0 ? 0 : given > most ? int32_t(most) : given;
            if (p.n_pages == 0u) t.length = 0;
            return t;
        }
        before += __shfl(upto, 63);
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

template <uint32_t D, uint32_t BITS>
__global__ __launch_bounds__(256) void attend_rows_kernel(AttendParams p) {
    constexpr uint32_t kKeyBytes = D * BITS / 32u, kValueBytes = D * BITS / 128u;      // of a key, of a value, that a lane feeds
    constexpr uint32_t kMfmas = D / 32u, kTiles = D / 16u, kVector = D * BITS / 8u;
    __shared__ float joined[kAttendWaves][kTileRows][D + 4u];
    __shared__ float stats[kAttendWaves][kTileRows][2];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, c = lane & 15u, g = lane >> 4;
    const uint32_t head = blockIdx.y, split = blockIdx.z;
    const Tile t = find_tile(p, blockIdx.x, kTileRows);
    if (t.n_rows == 0u) return;
    const int32_t seen = seen_by(p, t);
    const int32_t begin = int32_t(split * p.span), end = min(seen, begin + int32_t(p.span));
    const uint64_t part = (uint64_t(split) * p.n_tiles + blockIdx.x) * p.heads + head;
    if (p.splits > 1u && begin >= end) {                                                // nothing in this share
        if (threadIdx.x < kTileRows) reinterpret_cast<float2*>(p.part_stats)[part * kTileRows + threadIdx.x] = make_float2(-__builtin_inff(), 0.0f);
        return;
    }

    // the lane's part of query c, scaled into fp16
    const uint32_t row = t.first_row + min(c, t.n_rows - 1u), token = row / p.group, member = row - token * p.group;
    const int32_t position = t.length - int32_t(t.n_new) + int32_t(token);
    words4 q[kMfmas];
    float to_scores;
    {
        const uint16_t* from = p.q + uint64_t(t.first_token + token) * p.q_token_stride + uint64_t(head * p.group + member) * p.q_head_stride + g * (D / 4u);
        float v[kMfmas][8], most = 0.0f;
        for (uint32_t m = 0; m < kMfmas; ++m) {
            Eight<ANSZP_OUT_BF16> e;
            e.load(from, m * 8u, 8u);
            for (uint32_t j = 0; j < 8u; ++j) {
                v[m][j] = e[j];
                most = fmaxf(most, fabsf(e[j]));
            }
        }
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        const int32_t exponent = int32_t(__builtin_bit_cast(uint32_t, most) >> 23) - 127;
        const int32_t up = exponent == 128 ? 0 : min(13 - exponent, 126);
        const float factor = __builtin_bit_cast(float, uint32_t(up + 127) << 23);
        to_scores = p.scale * __builtin_bit_cast(float, uint32_t(127 - up) << 23);
        for (uint32_t m = 0; m < kMfmas; ++m) {
            // 4 bits: bytes of low halves, then of high ones
            constexpr uint32_t kOrder4[8] = {0, 2, 4, 6, 1, 3, 5, 7};
            f16x8 h;
            for (uint32_t j = 0; j < 8u; ++j) h[j] = static_cast<_Float16>(v[m][BITS == 4u ? kOrder4[j] : j] * factor);
            q[m] = __builtin_bit_cast(words4, h);
        }
    }

    floatx4 acc[kTiles] = {};
    float top = -__builtin_inff(), sum = 0.0f, reach = 0.0f;                            // m, the lane's part of l, the values' power of two
    for (int32_t t0 = begin + int32_t(wave * kStep); t0 < end; t0 += int32_t(kAttendWaves * kStep)) {
        floatx4 x[2];
        uint32_t hidden = 0u;                                                           // bit 4 u + i
        Bytes<kValueBytes> vb[2][4];
        float vs[2][4], vz[2][4];
        for (uint32_t u = 0; u < 2u; ++u) {
            const int32_t first = t0 + int32_t(16u * u);
            const bool inside = first < end;
            const uint32_t at = inside ? uint32_t(first) >> p.page_log : 0u;
            const int32_t named = p.pages[uint64_t(t.seq) * p.table_width + at];
            const bool there = inside && named >= 0 && uint64_t(named) < p.n_pages;
            if (inside && !there && lane == 0u) flag(p);
            const uint64_t base = ((uint64_t(there ? named : 0) * p.heads + head) << p.page_log) + (uint32_t(first) & ((1u << p.page_log) - 1u) & ~15u);
            // keys
            Bytes<kKeyBytes> kb;
            kb.load(p.k + (base + c) * kVector + g * kKeyBytes);
            float kz = p.k_params[2u * (base + c) + 1u];
            if (!there || first + int32_t(c) >= end) kz = 0.0f;
            const f16x2 offset = both(1024.0f + kz);
            floatx4 s = {0.0f, 0.0f, 0.0f, 0.0f};
            for (uint32_t m = 0; m < kMfmas; ++m) {
                words2 a, b;
                if constexpr (BITS == 8u) {
                    a = less_zero(kb.w[2u * m], offset);
                    b = less_zero(kb.w[2u * m + 1u], offset);
                } else {
                    a = less_zero(kb.w[m] & 0x0F0F0F0Fu, offset);
                    b = less_zero((kb.w[m] >> 4) & 0x0F0F0F0Fu, offset);
                }
                s = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, words4{a[0], a[1], b[0], b[1]}), __builtin_bit_cast(f16x8, q[m]), s, 0, 0, 0);
            }
            for (uint32_t i = 0; i < 4u; ++i) {
                const uint64_t n = base + g * 4u + i;
                const int32_t place = first + int32_t(g * 4u + i);
                vb[u][i].load(p.v + n * kVector + c * kValueBytes);
                const float2 w = reinterpret_cast<const float2*>(p.v_params)[n];
                const bool held = there && place < end;
                vs[u][i] = held ? w.x : 0.0f;
                vz[u][i] = held ? w.y : 0.0f;
                x[u][i] = s[i] * to_scores * p.k_params[2u * n];
                if (!held || place > position) {
                    x[u][i] = -__builtin_inff();
                    hidden |= 1u << (4u * u + i);
                }
            }
        }
        // running maximum, over the lane's tokens and the other lanes of the same query
        float high = top, far = reach;
        for (uint32_t u = 0; u < 2u; ++u)
            for (uint32_t i = 0; i < 4u; ++i) {
                high = fmaxf(high, x[u][i]);
                far = fmaxf(far, fabsf(vs[u][i]));
            }
        high = fmaxf(high, __shfl_xor(high, 16));
        high = fmaxf(high, __shfl_xor(high, 32));
        far = fmaxf(far, __shfl_xor(far, 16));
        far = fmaxf(far, __shfl_xor(far, 32));
        if (far > reach) far = __builtin_bit_cast(float, min((__builtin_bit_cast(uint32_t, far) + 0x7FFFFFu) & 0xFF800000u, 0x7E800000u));
        const float less = far > 0.0f ? 1.0f / far : 0.0f;
        const float safe = high == -__builtin_inff() ? 0.0f : high;
        const float kept = __builtin_amdgcn_exp2f(top - safe), kept_values = kept * (reach * less);
        top = high;
        reach = far;
        float l = 0.0f;
        words4 weights;
        for (uint32_t u = 0; u < 2u; ++u)
            for (uint32_t i = 0; i < 4u; i += 2u) {
                float w[2];
                for (uint32_t j = 0; j < 2u; ++j) {
                    const float e = __builtin_amdgcn_exp2f(x[u][i + j] - safe + 15.0f);
                    l += e;
                    w[j] = hidden >> (4u * u + i + j) & 1u ? 0.0f : e * (vs[u][i + j] * less);
                }
                weights[2u * u + i / 2u] = bits_of(f16x2{static_cast<_Float16>(w[0]), static_cast<_Float16>(w[1])});
            }
        sum = sum * kept + l;
        f16x2 z[4];
        for (uint32_t j = 0; j < 4u; ++j)
            z[j] = f16x2{static_cast<_Float16>(1024.0f + vz[j >> 1][2u * (j & 1u)]), static_cast<_Float16>(1024.0f + vz[j >> 1][2u * (j & 1u) + 1u])};
        for (uint32_t e = 0; e < kTiles; ++e) {
            words4 a;
            for (uint32_t j = 0; j < 4u; ++j) {
                const Bytes<kValueBytes>&one = vb[j >> 1][2u * (j & 1u)], &two = vb[j >> 1][2u * (j & 1u) + 1u];
                uint32_t pair;
                if constexpr (BITS == 8u) {
                    pair = __builtin_amdgcn_perm(two.w[e >> 2], one.w[e >> 2], 0x0C040C00u + (e & 3u) * 0x00010001u);
                } else {
                    pair = __builtin_amdgcn_perm(two.w[e >> 3], one.w[e >> 3], 0x0C040C00u + ((e & 7u) >> 1) * 0x00010001u);
                    pair = (e & 1u ? pair >> 4 : pair) & 0x000F000Fu;
                }
                a[j] = bits_of(halves(pair | 0x64006400u) - z[j]);
            }
            acc[e] *= kept_values;
            acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, weights), acc[e], 0, 0, 0);
        }
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);

    // the wavefronts' results together
    for (uint32_t e = 0; e < kTiles; ++e)
        for (uint32_t i = 0; i < 4u; ++i) joined[wave][c][(g * 4u + i) * kTiles + e] = acc[e][i] * reach;
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

// The splits' results together: a workgroup per tile and head, 16 threads a row.
template <uint32_t D>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendParams p) {
    constexpr uint32_t kMine = D / 16u;
    const uint32_t head = blockIdx.y;
    const Tile t = find_tile(p, blockIdx.x, kTileRows);
    const uint32_t r = threadIdx.x >> 4, d0 = (threadIdx.x & 15u) * kMine;
    if (r >= t.n_rows) return;
    const float2* stats = reinterpret_cast<const float2*>(p.part_stats);
    float high = -__builtin_inff(), l = 0.0f, o[kMine] = {};
    for (uint32_t s = 0; s < p.splits; ++s) high = fmaxf(high, stats[((uint64_t(s) * p.n_tiles + blockIdx.x) * p.heads + head) * kTileRows + r].x);
    const float safe = high == -__builtin_inff() ? 0.0f : high;
    for (uint32_t s = 0; s < p.splits; ++s) {
        const uint64_t part = ((uint64_t(s) * p.n_tiles + blockIdx.x) * p.heads + head) * kTileRows + r;
        const float2 w = stats[part];
        if (w.y == 0.0f) continue;
        const float by = __builtin_amdgcn_exp2f(w.x - safe);
        l += w.y * by;
        for (uint32_t d = 0; d < kMine; ++d) o[d] += p.parts[part * D + d0 + d] * by;
    }
    const float over = l == 0.0f ? 0.0f : 1.0f / l;
    const uint32_t row = t.first_row + r, token = row / p.group, member = row - token * p.group;
    const uint64_t to = uint64_t(t.first_token + token) * p.out_token_stride + uint64_t(head * p.group + member) * p.out_head_stride + d0;
    for (uint32_t d = 0; d < kMine; d += 4u) {
        const floatx4 v = {o[d] * over, o[d + 1u] * over, o[d + 2u] * over, o[d + 3u] * over};
        if (p.out_dtype == ANSZP_OUT_BF16)
            *reinterpret_cast<words2_any*>(static_cast<uint16_t*>(p.out) + to + d) = words2{to_bf16_pair(v[0], v[1]), to_bf16_pair(v[2], v[3])};
        else
            *reinterpret_cast<words4_any*>(static_cast<float*>(p.out) + to + d) = __builtin_bit_cast(words4, v);
    }
}

// How the tokens are shared out: enough workgroups for the chip, at least 256 tokens in each.
struct Shares {
    uint32_t tiles, splits, span;
};
Shares shares_of(const anszp_attend_args_t& a) {
    Shares s;
    s.tiles = static_cast<uint32_t>(a.n_tokens * a.group / kTileRows + a.n_seqs);
    const uint64_t most = uint64_t(a.table_width) * a.cache.page_size, groups = std::max<uint64_t>(1u, uint64_t(s.tiles) * a.cache.heads);
    uint64_t splits = std::min<uint64_t>(4u * device_cus() / groups, (most + 255u) / 256u);
    splits = std::max<uint64_t>(1u, std::min<uint64_t>(splits, 1024u));
    const uint64_t whole = kStep * kAttendWaves;
    s.span = static_cast<uint32_t>((most + splits * whole - 1u) / (splits * whole) * whole);
    s.splits = static_cast<uint32_t>((most + s.span - 1u) / s.span);
    return s;
}

bool in_range(const anszp_attend_args_t& a) {
    const anszp_cache_t& c = a.cache;
    return !(a.n_tokens >= 1u << 24 || a.n_seqs >= 1u << 24 || a.table_width == 0u || uint64_t(a.table_width) * c.page_size > 1ull << 30 || a.group == 0u ||
             a.group > 256u || (a.out_dtype != ANSZP_OUT_F32 && a.out_dtype != ANSZP_OUT_BF16) || a.n_tokens * a.group / kTileRows + a.n_seqs >= 1ull << 31);
}

uint64_t workspace_of(const anszp_attend_args_t& a, const Shares& s) {
    return s.splits > 1u ? uint64_t(s.splits) * s.tiles * a.cache.heads * kTileRows * (a.cache.head_dim + 2u) * sizeof(float) : 0u;
}

template <uint32_t D>
void launch(const AttendParams& p, uint32_t bits, hipStream_t s) {
    const dim3 grid(p.n_tiles, p.heads, p.splits);
    if (bits == 8u) hipLaunchKernelGGL((attend_rows_kernel<D, 8u>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((attend_rows_kernel<D, 4u>), grid, dim3(256), 0, s, p);
    if (p.splits > 1u) hipLaunchKernelGGL(attend_join_kernel<D>, dim3(p.n_tiles, p.heads), dim3(256), 0, s, p);
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
    const Shares s = shares_of(*a);
    const uint64_t need = workspace_of(*a, s);
    if (need && !a->workspace) return ANSZP_E_NULL;
    if (a->workspace_bytes < need || (reinterpret_cast<uintptr_t>(a->workspace) & 15u)) return ANSZP_E_RANGE;
    AttendParams p = {};
    p.k = a->cache.k; p.k_params = a->cache.k_params; p.v = a->cache.v; p.v_params = a->cache.v_params;
    p.q = static_cast<const uint16_t*>(a->q); p.out = a->out; p.pages = a->pages; p.lengths = a->lengths; p.starts = a->starts; p.status = a->status;
    p.parts = static_cast<float*>(a->workspace);
    p.part_stats = p.parts + uint64_t(s.splits) * s.tiles * a->cache.heads * kTileRows * a->cache.head_dim;
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
