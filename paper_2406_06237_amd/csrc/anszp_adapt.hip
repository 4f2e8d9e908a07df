// Low-rank adapters of many requests beside a shared product, for gfx950: with i = ids[r], the adapter of row r,
//   h = scales[i] * x_scales[r] * a[i] x[r]              out = act(base + b[i] h) * mul + residual
// and no adapter's part for ids below 0.  Two launches: h from all of k, then the output's columns.
//
// Rows come in tiles of 16, and a tile is worked through once for each adapter that its rows have: one for a prompt, up to sixteen for a step of as
// many requests.  What a row has from other rows' adapters is never selected, so that nothing in them, an infinity or a NaN, reaches it.  x and a are bf16 (8-bit rows are exact in
// it), their sums in 32 bits.  h goes into the second product as two bf16 numbers, to 2^-18 of it, for bf16 outputs, and as three, all of it, for fp32 ones: a number rounded
// to bf16 leaves a rest that is exact.
//
// Memory bounds it: base and out once, x once, the adapters that are there.
#include <hip/hip_runtime.h>

#include "anszp_cus.h"
#include "anszp_epilogue.h"
#include "anszp_numbers.h"

namespace {

struct AdaptParams {
    const uint8_t* x;
    const uint16_t* a;
    const uint16_t* b;
    const int32_t* ids;
    const float* x_scales;
    const float* scales;
    const void* base;
    const void* mul;
    const void* residual;
    void* out;
    float* h;                           // [part of k][row][rank up to a multiple of 8]
    uint32_t* status;
    uint64_t x_stride, a_stride, a_row_stride, b_stride, b_row_stride, base_stride, mul_stride, residual_stride, out_stride;    // x's in bytes
    uint64_t rows, cols;
    uint32_t adapters, k, rank, rank_room, base_dtype, out_dtype, activation;
    uint32_t slots, groups, parts;      // workgroups that share a tile's adapters, groups of ranks, parts of k
    uint32_t blocks, terms;             // blocks of 8 ranks a term of h has, terms
    uint32_t across;                    // workgroups that a row's columns take
};

__device__ __forceinline__ bf16x8 as_bf16(words4 w) { return __builtin_bit_cast(bf16x8, w); }

// Sixteen consecutive elements of a row of bf16 or of signed bytes, as two operands; zeros behind its end.
template <bool BYTES>
struct Sixteen {
    words4 lo, hi;
    __device__ __forceinline__ void load(const uint8_t* row, uint32_t at, uint32_t there) {
        if constexpr (BYTES) {
            const uint8_t* p = row + at;
            hi = words4{0u, 0u, 0u, 0u};
            if (there >= 16u) {
                lo = *reinterpret_cast<const words4_any*>(p);
            } else {
                lo = words4{0u, 0u, 0u, 0u};
                for (uint32_t i = 0; i < 16u; ++i)
                    if (i < there) lo[i >> 2] |= uint32_t(p[i]) << (8u * (i & 3u));
            }
        } else {
            const uint16_t* p = reinterpret_cast<const uint16_t*>(row) + at;
            Eight<ANSZP_OUT_BF16> a, b;
            a.load(p, 0u, there);
            b.load(p, 8u, there > 8u ? there - 8u : 0u);
            lo = a.w;
            hi = b.w;
        }
    }
    // A whole number below 2^8 in size fits bf16, so the upper half of its binary32 is all of it.
    __device__ __forceinline__ bf16x8 operand(uint32_t half) const {
        if constexpr (BYTES) {
            words4 w;
            for (uint32_t i = 0; i < 4u; ++i) {
                const uint32_t four = lo[half * 2u + (i >> 1)], at = 16u * (i & 1u);
                const float a = float(int32_t(four << (24u - at)) >> 24), b = float(int32_t(four << (16u - at)) >> 24);
                w[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302u);
            }
            return as_bf16(w);
        } else {
            return as_bf16(half ? hi : lo);
        }
    }
};

__device__ __forceinline__ int32_t id_of(const AdaptParams& p, uint64_t row, bool tells) {
    if (row >= p.rows) return -1;
    const int32_t id = p.ids[row];
    if (id < 0 || uint32_t(id) < p.adapters) return id;
    if (tells && p.status) {
        atomicOr(&p.status[0], ANSZP_ST_BAD_DESC);
        atomicAdd(&p.status[1], 1u);
    }
    return -1;
}

// work(adapter, lanes that have it) for each adapter that the first `n` lanes' rows have.
template <class Work>
__device__ __forceinline__ void each_adapter(int32_t id, uint32_t n, Work work) {
    uint64_t left = __ballot(id >= 0 && (threadIdx.x & 63u) < n);
    while (left) {
        const int32_t one = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        const uint64_t same = __ballot(id == one) & left;
        left &= ~same;
        work(uint32_t(one), same);
    }
}

// h of 16 rows and up to 16 * RANKS ranks.  ROWS: a wavefront has a tile of rows of its own; else the four of a workgroup share a tile's k.
template <bool BYTES, bool ROWS, uint32_t RANKS>
__global__ __launch_bounds__(256) void adapt_down_kernel(AdaptParams p) {
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, c = lane & 15u, g = lane >> 4;
    const uint32_t slot = blockIdx.y / p.groups, group = blockIdx.y - slot * p.groups, part = blockIdx.z;
    const uint64_t first = (uint64_t(blockIdx.x) * (ROWS ? 4u : 1u) + (ROWS ? wave : 0u)) * 16u;
    if (ROWS && first >= p.rows) return;
    const int32_t id = id_of(p, first + c, false);
    const uint32_t steps = (p.k + 63u) / 64u, share = ROWS ? part : part * 4u + wave, shares = ROWS ? p.parts : p.parts * 4u;
    const uint32_t begin = uint32_t(uint64_t(steps) * share / shares), end = uint32_t(uint64_t(steps) * (share + 1u) / shares);
    const uint64_t row = least(first + c, p.rows - 1u);
    const uint8_t* const x = p.x + row * p.x_stride;
    __shared__ floatx4 sums[ROWS ? 1u : 4u][ROWS ? 1u : RANKS][64];
    uint32_t turn = 0u;
    each_adapter(id, 16u, [&](uint32_t one, uint64_t) __attribute__((always_inline)) {
        if (turn++ % p.slots != slot) return;
        const uint16_t* a[RANKS];
        for (uint32_t t = 0; t < RANKS; ++t) a[t] = p.a + one * p.a_stride + least((group * RANKS + t) * 16u + c, p.rank - 1u) * p.a_row_stride;
        floatx4 sum[RANKS] = {};
        const auto step = [&](uint32_t s) __attribute__((always_inline)) {
            const uint32_t at = s * 64u + g * 16u, there = at < p.k ? p.k - at : 0u;
            Sixteen<BYTES> xs;
            Sixteen<false> as[RANKS];
            xs.load(x, at, there);
            for (uint32_t t = 0; t < RANKS; ++t) as[t].load(reinterpret_cast<const uint8_t*>(a[t]), at, there);
            for (uint32_t half = 0; half < 2u; ++half)
                for (uint32_t t = 0; t < RANKS; ++t) sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xs.operand(half), as[t].operand(half), sum[t], 0, 0, 0);
        };
        for (uint32_t s = begin; s < end; ++s) step(s);
        if constexpr (!ROWS) {
            __syncthreads();
            for (uint32_t t = 0; t < RANKS; ++t) sums[wave][t][lane] = sum[t];
            __syncthreads();
            if (wave != 0u) return;
            for (uint32_t w = 1; w < 4u; ++w)
                for (uint32_t t = 0; t < RANKS; ++t) sum[t] += sums[w][t][lane];
        }
        const float by = p.scales ? p.scales[one] : 1.0f;
        for (uint32_t i = 0; i < 4u; ++i) {
            const uint32_t n = 4u * g + i;
            if (__shfl(id, n) != int32_t(one)) continue;
            const float scale = p.x_scales ? by * p.x_scales[first + n] : by;
            for (uint32_t t = 0; t < RANKS; ++t) {
                const uint32_t rank = (group * RANKS + t) * 16u + c;
                if (rank < p.rank) p.h[(part * p.rows + first + n) * p.rank_room + rank] = scale * sum[t][i];
            }
        }
    });
}

// The nearest bf16 (of a number that would become infinite the one below it, so that what is left is a number).
__device__ __forceinline__ uint16_t part_of(float h) {
    return !(__builtin_fabsf(h) < 0x1p127f) ? uint16_t(__builtin_bit_cast(uint32_t, h) >> 16) | (h != h ? 0x40u : 0u) : to_bf16(h);
}

// 64 columns a wavefront, 16 * TILES rows a workgroup.  In the instructions' terms b's rows are the rows, in an order that leaves each lane with 16
// consecutive columns of its row.
template <uint32_t TILES>
__global__ __launch_bounds__(256) void adapt_up_kernel(AdaptParams p) {
    extern __shared__ __attribute__((aligned(16))) uint16_t terms_of_h[];                           // [row][term][block][8], 8 more behind a row
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, c = lane & 15u, g = lane >> 4;
    const uint32_t tile = blockIdx.x / p.across, piece = blockIdx.x - tile * p.across;
    const uint64_t first = uint64_t(tile) * (16u * TILES), from = uint64_t(piece) * 256u + wave * 64u;
    const uint32_t steps = (p.blocks * p.terms + 3u) / 4u, width = steps * 32u + 8u;
    const int32_t id = id_of(p, first + (lane & (16u * TILES - 1u)), piece == 0u && wave == 0u && lane < 16u * TILES);
    for (uint32_t n = threadIdx.x; n < 16u * TILES * steps * 32u; n += 256u) {
        const uint32_t r = n / (steps * 32u), at = n - r * (steps * 32u), block = at / 8u, term = block / p.blocks, rank = (block - term * p.blocks) * 8u + (at & 7u);
        float h = 0.0f;
        if (first + r < p.rows && rank < p.rank && term < p.terms) {
            const int32_t own = p.ids[first + r];
            if (own >= 0 && uint32_t(own) < p.adapters)
                for (uint32_t s = 0; s < p.parts; ++s) h += p.h[(s * p.rows + first + r) * p.rank_room + rank];
            for (uint32_t t = 0; t < term; ++t) h = __builtin_fabsf(h) < __builtin_inff() ? h - bf16_low(part_of(h)) : 0.0f;
        }
        terms_of_h[r * width + at] = part_of(h);
    }
    __syncthreads();
    if (from >= p.cols) return;
    int32_t own[TILES];
    for (uint32_t r = 0; r < TILES; ++r) own[r] = __shfl(id, r * 16u + c);
    floatx4 sum[TILES][4] = {};
    each_adapter(id, 16u * TILES, [&](uint32_t one, uint64_t lanes) __attribute__((always_inline)) {
        floatx4 part[TILES][4] = {};
        const uint16_t* b[4];
        for (uint32_t t = 0; t < 4u; ++t) b[t] = p.b + one * p.b_stride + least(from + (c >> 2) * 16u + t * 4u + (c & 3u), p.cols - 1u) * p.b_row_stride;
        for (uint32_t s = 0; s < steps; ++s) {
            const uint32_t block = (s * 4u + g) % p.blocks * 8u, there = block < p.rank ? p.rank - block : 0u;
            Eight<ANSZP_OUT_BF16> w[4];
            for (uint32_t t = 0; t < 4u; ++t) w[t].load(b[t], block, there);
            for (uint32_t r = 0; r < TILES; ++r) {
                if (!(lanes >> (16u * r) & 0xFFFFu)) continue;
                const bf16x8 h = *reinterpret_cast<const bf16x8*>(terms_of_h + (r * 16u + c) * width + s * 32u + g * 8u);
                for (uint32_t t = 0; t < 4u; ++t) part[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(w[t].w), h, part[r][t], 0, 0, 0);
            }
        }
        for (uint32_t r = 0; r < TILES; ++r)
            for (uint32_t t = 0; t < 4u; ++t) sum[r][t] = own[r] == int32_t(one) ? part[r][t] : sum[r][t];
    });
    for (uint32_t r = 0; r < TILES; ++r) {
        const uint64_t row = first + r * 16u + c;
        if (row >= p.rows) continue;
        for (uint32_t half = 0; half < 2u; ++half) {
            const uint64_t col = from + g * 16u + half * 8u;
            if (col >= p.cols) continue;
            const uint32_t there = p.cols - col < 8u ? uint32_t(p.cols - col) : 8u;
            Some<8u> base, mul, residual;
            base.load(p.base, p.base_dtype, row * p.base_stride + col, there);
            if (p.mul) mul.load(p.mul, p.out_dtype, row * p.mul_stride + col, there);
            if (p.residual) residual.load(p.residual, p.out_dtype, row * p.residual_stride + col, there);
            float v[8];
            for (uint32_t i = 0; i < 8u; ++i) {
                v[i] = base.at(p.base_dtype, i);
                if (own[r] >= 0) v[i] += sum[r][half * 2u + (i >> 2)][i & 3u];
                v[i] = activated(v[i], p.activation);
                if (p.mul) v[i] *= mul.at(p.out_dtype, i);
                if (p.residual) v[i] += residual.at(p.out_dtype, i);
            }
            store_eight(p.out, p.out_dtype, row * p.out_stride + col, there, v);
        }
    }
}

struct Plan {
    bool rows;                          // a wavefront a tile of rows
    uint32_t ranks;                     // 16s of ranks a workgroup has
    uint32_t slots, groups, parts;
    uint64_t workspace;
};

int adapt_check(const anszp_adapt_args_t& a) {
    if ((a.x_dtype != ANSZP_OUT_BF16 && a.x_dtype != ANSZP_I8) || (a.base_dtype != ANSZP_OUT_F32 && a.base_dtype != ANSZP_OUT_BF16) ||
        (a.out_dtype != ANSZP_OUT_F32 && a.out_dtype != ANSZP_OUT_BF16) || a.activation > ANSZP_FN_SILU || a.k == 0 || a.k > 1u << 30 || a.rank == 0 || a.rank > 256u ||
        a.rows >= 1ull << 28 || a.cols >= 1ull << 31 || a.adapters >= 1u << 24)
        return ANSZP_E_RANGE;
    if (a.rows > 1 && a.out_stride < a.cols) return ANSZP_E_RANGE;
    return ANSZP_OK;
}

Plan plan_of(const anszp_adapt_args_t& a) {
    Plan q = {};
    if (a.adapters == 0u) return q;
    const uint32_t tiles = static_cast<uint32_t>((a.rows + 15u) / 16u), steps = (a.k + 63u) / 64u, sixteens = (a.rank + 15u) / 16u;
    q.ranks = sixteens <= 1u ? 1u : sixteens <= 2u ? 2u : 4u;
    q.groups = (sixteens + q.ranks - 1u) / q.ranks;
    q.rows = tiles >= 64u;
    q.slots = q.rows ? 1u : static_cast<uint32_t>(a.rows < 16u ? a.rows : 16u);
    if (q.slots > a.adapters) q.slots = a.adapters;
    const uint32_t groups = (q.rows ? (tiles + 3u) / 4u : tiles * q.slots) * q.groups, most = q.rows ? (steps + 3u) / 4u : (steps + 7u) / 8u;
    q.parts = (2u * device_cus() + groups - 1u) / groups;
    if (q.parts > 16u) q.parts = 16u;
    if (q.parts > most) q.parts = most;
    q.workspace = (q.parts * a.rows * ((a.rank + 7u) / 8u * 8u) * 4u + 15u) & ~15ull;
    return q;
}

template <bool BYTES, bool ROWS>
void launch_down(const AdaptParams& p, const Plan& q, hipStream_t s) {
    const uint32_t tiles = static_cast<uint32_t>((p.rows + 15u) / 16u);
    const dim3 grid(ROWS ? (tiles + 3u) / 4u : tiles, q.slots * q.groups, q.parts), threads(256);
    if (q.ranks == 1u) hipLaunchKernelGGL((adapt_down_kernel<BYTES, ROWS, 1u>), grid, threads, 0, s, p);
    else if (q.ranks == 2u) hipLaunchKernelGGL((adapt_down_kernel<BYTES, ROWS, 2u>), grid, threads, 0, s, p);
    else hipLaunchKernelGGL((adapt_down_kernel<BYTES, ROWS, 4u>), grid, threads, 0, s, p);
}

}  // namespace

extern "C" uint64_t anszp_adapt_workspace_bytes(const anszp_adapt_args_t* a) {
    return !a || adapt_check(*a) || a->rows == 0 || a->cols == 0 ? 0u : plan_of(*a).workspace;
}

extern "C" int anszp_adapt(const anszp_adapt_args_t* a, void* hip_stream) {
    if (!a) return ANSZP_E_NULL;
    const int rc = adapt_check(*a);
    if (rc) return rc;
    if (a->rows == 0 || a->cols == 0) return ANSZP_OK;
    if (!a->base || !a->out || !a->ids || (a->adapters && (!a->x || !a->a || !a->b))) return ANSZP_E_NULL;
    const bool bytes = a->x_dtype == ANSZP_I8;
    const uint64_t size = a->out_dtype == ANSZP_OUT_BF16 ? 2u : 4u, base_size = a->base_dtype == ANSZP_OUT_BF16 ? 2u : 4u, x_size = bytes ? 1u : 2u, width = a->cols * size;
    const Rows out = {a->out, a->rows, a->out_stride * size, width}, base = {a->base, a->rows, a->base_stride * base_size, a->cols * base_size};
    if (meet(out, {a->x_scales, 1, 0, a->rows * 4u}) || meet(out, {a->scales, 1, 0, a->adapters * 4u}) || meet(out, {a->x, a->rows, a->x_stride * x_size, a->k * x_size}) || meet(out, {a->ids, 1, 0, a->rows * 4u}) ||
        (base_size == size ? meet_elsewhere(out, base) : meet(out, base)) || meet_elsewhere(out, {a->mul, a->rows, a->mul_stride * size, width}) ||
        meet_elsewhere(out, {a->residual, a->rows, a->residual_stride * size, width}) ||
        meet(out, {a->a, 1, 0, ((a->adapters - 1ull) * a->a_stride + (a->rank - 1ull) * a->a_row_stride + a->k) * (a->adapters ? 2u : 0u)}) ||
        meet(out, {a->b, 1, 0, ((a->adapters - 1ull) * a->b_stride + (a->cols - 1ull) * a->b_row_stride + a->rank) * (a->adapters ? 2u : 0u)}))
        return ANSZP_E_RANGE;
    if ((a->rows + 15u) / 16u * ((a->cols + 255u) / 256u) >= 1ull << 24) return ANSZP_E_RANGE;          // (threads that one launch has not)
    const Plan q = plan_of(*a);
    if (q.workspace && !a->workspace) return ANSZP_E_NULL;
    if (q.workspace && (a->workspace_bytes < q.workspace || (reinterpret_cast<uintptr_t>(a->workspace) & 15u))) return ANSZP_E_RANGE;
    AdaptParams p = {};
    p.x = static_cast<const uint8_t*>(a->x); p.a = static_cast<const uint16_t*>(a->a); p.b = static_cast<const uint16_t*>(a->b);
    p.ids = a->ids; p.x_scales = a->x_scales; p.scales = a->scales; p.base = a->base; p.mul = a->mul; p.residual = a->residual; p.out = a->out;
    p.h = static_cast<float*>(a->workspace); p.status = a->status;
    p.x_stride = a->x_stride * x_size; p.a_stride = a->a_stride; p.a_row_stride = a->a_row_stride; p.b_stride = a->b_stride; p.b_row_stride = a->b_row_stride;
    p.base_stride = a->base_stride; p.mul_stride = a->mul_stride; p.residual_stride = a->residual_stride; p.out_stride = a->out_stride;
    p.rows = a->rows; p.cols = a->cols; p.adapters = a->adapters; p.k = a->k; p.rank = a->rank; p.rank_room = (a->rank + 7u) / 8u * 8u;
    p.base_dtype = a->base_dtype; p.out_dtype = a->out_dtype; p.activation = a->activation;
    p.slots = q.slots; p.groups = q.groups; p.parts = q.parts;
    p.across = static_cast<uint32_t>((a->cols + 255u) / 256u);
    const uint32_t blocks = (a->rank + 7u) / 8u;
    p.terms = a->out_dtype == ANSZP_OUT_BF16 ? 2u : 3u;
    p.blocks = blocks <= 2u ? blocks : (blocks + 3u) / 4u * 4u;     // (a step of the second product has four blocks: of one term, or of several short ones)
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (q.workspace) {
        if (bytes && q.rows) launch_down<true, true>(p, q, s);
        else if (bytes) launch_down<true, false>(p, q, s);
        else if (q.rows) launch_down<false, true>(p, q, s);
        else launch_down<false, false>(p, q, s);
    }
    const uint32_t row_bytes = ((p.blocks * p.terms + 3u) / 4u * 32u + 8u) * 2u;
    if (a->rows >= 1024u && 64u * row_bytes <= 65536u) hipLaunchKernelGGL(adapt_up_kernel<4u>, dim3(p.across * static_cast<uint32_t>((a->rows + 63u) / 64u)), dim3(256), 64u * row_bytes, s, p);
    else hipLaunchKernelGGL(adapt_up_kernel<1u>, dim3(p.across * static_cast<uint32_t>((a->rows + 15u) / 16u)), dim3(256), 16u * row_bytes, s, p);
    return hipGetLastError() == hipSuccess ? ANSZP_OK : ANSZP_E_HIP;
}
