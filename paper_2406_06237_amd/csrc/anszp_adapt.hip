// Low-rank adapters of many requests beside a shared product, for gfx950: with i = ids[r], the adapter of row r,
//   h = scales[i] * x_scales[r] * a[i] x[r]              out = act(base + b[i] h) * mul + residual
// and no adapter's part for ids below 0.  Two launches: h from all of k, then the output's columns.
//
// Rows come in tiles of 64, and a tile is worked through once for each adapter that its rows have: one for a prompt, up to 64 for a step of as
// many requests.  What a row has from other rows' adapters is never selected, so that nothing in them, an infinity or a NaN, reaches it.  x and a are bf16
// (8-bit rows are exact in it), their sums in 32 bits.  h goes into the second product as three bf16 numbers of 8 bits each, which are all
// of it.  (Two, rounded, are up to 2^-18 off, and where base or residual cancels the sum that is several steps of a bf16 output.)
//
// Memory bounds it: base and out once, x once, the adapters that are there.  8192 rows of 4096 bytes to 11008 columns in bf16 with rank 64, silu and mul: h
// 24 to 27 us (1.3 TB/s of x, 170 TFLOP/s), its terms 5, the columns 134 to 148 (4 TB/s, the vector unit busy 56 % of the time; torch's product of two such
// matrices, which streams as many bytes, 92).  1531 rows from 11008 bf16 to 4096 fp32 with a residual, rank 24: 15, 5 and 18 (4 TB/s).  64 requests with 48
// adapters of rank 16: 6.5 and 14 us, most of them waiting for loads: each workgroup of the second product adds up the parts of h of its 64 rows first.
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
    uint16_t* terms_of_h;               // of many rows, [row][width]
    uint32_t* status;
    uint64_t x_stride, a_stride, a_row_stride, b_stride, b_row_stride, base_stride, mul_stride, residual_stride, out_stride;    // x's in bytes
    uint64_t rows, cols;
    uint32_t adapters, k, rank, rank_room, activation;
    uint32_t slots, groups, parts;      // workgroups that share a tile's rows, groups of ranks, parts of k
    uint32_t blocks;                    // of 8 ranks that a term of h has
    uint32_t across, width;             // workgroups that a row's columns take; a row of h's terms
    const uint8_t* x_last;              // where the last 16 bytes of each begin
    const uint8_t* a_last;
    const uint8_t* b_last;
};

constexpr uint32_t kTerms = 3;          // bf16 numbers that are one of h

__device__ __forceinline__ bf16x8 as_bf16(words4 w) { return __builtin_bit_cast(bf16x8, w); }

// The first `there` bytes of 16 (0 and below: none), zeros behind them.
__device__ __forceinline__ words4 first_bytes(words4 w, int32_t there) {
#pragma unroll
    for (int32_t i = 0; i < 4; ++i) {
        const int32_t n = there - 4 * i;
        w[i] &= n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
    }
    return w;
}
// 16 bytes of which the first `there` are an operand's, whose last 16 begin at `last`: nothing behind them is read, and what lies between its rows counts as zeros.
// (Ends of rows one element at a time take a way of the program each, and so many registers that few wavefronts are left.)
__device__ __forceinline__ words4 careful(const uint8_t* at, int32_t there, const uint8_t* last) {
    const uint64_t over = at > last ? uint64_t(at - last) : 0u;
    const words4 w = *reinterpret_cast<const words4_any*>(at - over);
    uint64_t lo = uint64_t(w[1]) << 32 | w[0], hi = uint64_t(w[3]) << 32 | w[2];
    const uint32_t by = uint32_t(over < 16u ? over : 16u) * 8u;
    lo = by >= 64u ? (by >= 128u ? 0u : hi >> (by - 64u)) : by ? lo >> by | hi << (64u - by) : lo;
    hi = by >= 64u ? 0u : hi >> by;
    return first_bytes(words4{uint32_t(lo), uint32_t(lo >> 32), uint32_t(hi), uint32_t(hi >> 32)}, there);
}

// Eight signed bytes as an operand.  A whole number below 2^8 in size fits bf16, so the upper half of its binary32 is all of it.
__device__ __forceinline__ bf16x8 bf16_of_bytes(words2 bytes) {
    words4 w;
#pragma unroll
    for (uint32_t i = 0; i < 4u; ++i) {
        const uint32_t four = bytes[i >> 1], at = 16u * (i & 1u);
        const float lo = float(int32_t(four << (24u - at)) >> 24), hi = float(int32_t(four << (16u - at)) >> 24);
        w[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
    }
    return as_bf16(w);
}

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

// The adapters that a tile of 64 rows has, one after the other, by the lanes (a row each) that have them.
struct Adapters {
    int32_t id;
    uint64_t left, lanes;
    __device__ __forceinline__ explicit Adapters(int32_t of_row) : id(of_row), left(__ballot(of_row >= 0)), lanes(0u) {}
    // the next one, or -1
    __device__ __forceinline__ int32_t next() {
        if (!left) return -1;
        const int32_t one = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        lanes = __ballot(id == one);
        left &= ~lanes;
        return one;
    }
};

// h of 64 rows and up to 16 * RANKS ranks, 16 rows a wavefront.  128 or 256 bytes of each row of x and as much of k of a's rows go to LDS at a time, in
// pieces of 16 bytes end to end (operands taken from memory as the instructions want them are 16 bytes of 16 rows for every 16 lanes, and a CU looks up four
// times the lines: 33 us for 8192 rows of 4096 bytes and rank 64, this 25); two times of them are under way beside the one in LDS.
constexpr uint32_t at_once(bool bytes, uint32_t ranks) { return bytes || ranks <= 2u ? 128u : 64u; }
template <bool BYTES, uint32_t RANKS>
__global__ __launch_bounds__(256, 3) void adapt_down_kernel(AdaptParams p) {
    constexpr uint32_t kAtOnce = at_once(BYTES, RANKS), kRowOfX = kAtOnce * (BYTES ? 1u : 2u), kRowOfA = kAtOnce * 2u, kInX = kRowOfX / 16u, kInA = kRowOfA / 16u;
    constexpr uint32_t kPiecesOfA = RANKS * 16u * kInA, kEachOfA = (kPiecesOfA + 255u) / 256u, kEachOfX = 64u * kInX / 256u;
    __shared__ __attribute__((aligned(16))) uint8_t xs[2][64][kRowOfX + 16u], as[2][16u * RANKS][kRowOfA + 16u];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, c = lane & 15u, g = lane >> 4;
    const uint32_t slot = blockIdx.y / p.groups, group = blockIdx.y - slot * p.groups, part = blockIdx.z;
    const uint64_t first = uint64_t(blockIdx.x) * 64u;
    const uint32_t steps = (p.k + kAtOnce - 1u) / kAtOnce, begin = uint32_t(uint64_t(steps) * part / p.parts), end = uint32_t(uint64_t(steps) * (part + 1u) / p.parts);
    const float x_scale = p.x_scales ? p.x_scales[least(first + lane, p.rows - 1u)] : 1.0f;
    const int32_t id = id_of(p, first + lane, false);
    // This thread's pieces are every 256th of x's and of a's.
    const uint32_t x_row = threadIdx.x / kInX, x_piece = threadIdx.x % kInX * 16u;
    constexpr uint32_t kRowsApart = 256u / kInX;
    // Few rows: a workgroup for each, which works at the row's adapter if no row before has it.  Else the adapters in turn.
    uint64_t left = __ballot(id >= 0);
    uint32_t wait = slot;
    if (p.slots >= p.rows || p.slots == 64u) {
        const int32_t one = __builtin_amdgcn_readlane(id, slot);
        const uint64_t lanes = __ballot(id == one);
        left = one >= 0 && uint32_t(__builtin_ctzll(lanes)) == slot ? lanes : 0u;
        wait = 0u;
    }
    while (left) {
        const int32_t one = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        const uint64_t lanes = __ballot(id == one);
        left &= ~lanes;
        if (wait) {
            --wait;
            continue;
        }
        wait = p.slots - 1u;
        const float by = p.scales ? p.scales[one] : 1.0f;
        const uint8_t* x[kEachOfX];
        const uint8_t* a[kEachOfA];
        bool has[kEachOfX];
#pragma unroll
        for (uint32_t i = 0; i < kEachOfX; ++i) {
            has[i] = lanes >> (x_row + kRowsApart * i) & 1u;               // (rows of other adapters stay what they were: nothing of theirs is kept)
            x[i] = p.x + least(first + x_row + kRowsApart * i, p.rows - 1u) * p.x_stride + x_piece;
        }
#pragma unroll
        for (uint32_t i = 0; i < kEachOfA; ++i) {
            const uint32_t n = threadIdx.x + i * 256u;
            a[i] = reinterpret_cast<const uint8_t*>(p.a + uint64_t(one) * p.a_stride + least(group * RANKS * 16u + n / kInA, p.rank - 1u) * p.a_row_stride) + n % kInA * 16u;
        }
        struct Step {
            words4 x[kEachOfX], a[kEachOfA];
        } now, then;
        const auto load = [&](Step& to, uint32_t s) __attribute__((always_inline)) {
            if (s * kAtOnce + kAtOnce <= p.k) {
#pragma unroll
                for (uint32_t i = 0; i < kEachOfA; ++i) to.a[i] = *reinterpret_cast<const words4_any*>(a[i] + uint64_t(s) * kRowOfA);
#pragma unroll
                for (uint32_t i = 0; i < kEachOfX; ++i)
                    if (has[i]) to.x[i] = *reinterpret_cast<const words4_any*>(x[i] + uint64_t(s) * kRowOfX);
            } else {
                const int32_t left = int32_t(p.k - s * kAtOnce);
#pragma unroll
                for (uint32_t i = 0; i < kEachOfA; ++i)
                    to.a[i] = careful(a[i] + uint64_t(s) * kRowOfA, left * 2 - int32_t((threadIdx.x + i * 256u) % kInA * 16u), p.a_last);
#pragma unroll
                for (uint32_t i = 0; i < kEachOfX; ++i)
                    if (has[i]) to.x[i] = careful(x[i] + uint64_t(s) * kRowOfX, left * (BYTES ? 1 : 2) - int32_t(x_piece), p.x_last);
            }
        };
        floatx4 sum[RANKS] = {};
        const bool works = (lanes >> (16u * wave) & 0xFFFFu) != 0u;
        const auto step = [&](const Step& with, uint32_t s, Step& next) __attribute__((always_inline)) {
            const uint32_t buffer = (s - begin) & 1u;
#pragma unroll
            for (uint32_t i = 0; i < kEachOfA; ++i) {
                const uint32_t n = threadIdx.x + i * 256u;
                if (kPiecesOfA % 256u == 0u || n < kPiecesOfA) *reinterpret_cast<words4*>(&as[buffer][n / kInA][n % kInA * 16u]) = with.a[i];
            }
#pragma unroll
            for (uint32_t i = 0; i < kEachOfX; ++i)
                if (has[i]) *reinterpret_cast<words4*>(&xs[buffer][x_row + kRowsApart * i][x_piece]) = with.x[i];
            __syncthreads();
            if (s + 2u < end) load(next, s + 2u);
            if (!works) return;
#pragma unroll
            for (uint32_t k = 0; k < kAtOnce; k += 32u) {
                bf16x8 of_x;
                if constexpr (BYTES) of_x = bf16_of_bytes(*reinterpret_cast<const words2*>(&xs[buffer][wave * 16u + c][k + g * 8u]));
                else of_x = as_bf16(*reinterpret_cast<const words4*>(&xs[buffer][wave * 16u + c][(k + g * 8u) * 2u]));
#pragma unroll
                for (uint32_t t = 0; t < RANKS; ++t)
                    sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(of_x, as_bf16(*reinterpret_cast<const words4*>(&as[buffer][t * 16u + c][(k + g * 8u) * 2u])), sum[t], 0, 0, 0);
            }
        };
        if (begin < end) load(now, begin);
        if (begin + 1u < end) load(then, begin + 1u);
        for (uint32_t s = begin; s < end; s += 2u) {
            step(now, s, now);
            if (s + 1u < end) step(then, s + 1u, then);
        }
        // (the next adapter's first step goes to the buffer that this one's last may still be read from)
        __syncthreads();
        if (!works) continue;
#pragma unroll
        for (uint32_t i = 0; i < 4u; ++i) {
            const uint32_t n = wave * 16u + 4u * g + i;
            const float scale = by * __shfl(x_scale, n);
            if (!(lanes >> n & 1u)) continue;
#pragma unroll
            for (uint32_t t = 0; t < RANKS; ++t) {
                const uint32_t rank = (group * RANKS + t) * 16u + c;
                if (rank < p.rank) p.h[(part * p.rows + first + n) * p.rank_room + rank] = scale * sum[t][i];
            }
        }
    }
}

// Eight ranks of h of a row, the parts of k added up; what a row without an adapter has there is not looked at.
template <uint32_t AT_ONCE>
__device__ __forceinline__ void load_h(const AdaptParams& p, uint64_t row, uint32_t block, float (&h)[8]) {
    const float* const from = p.h + row * p.rank_room + block * 8u;
    const uint64_t apart = p.rows * p.rank_room;
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) h[i] = 0.0f;
    // (several under way together; behind the last one it is read again, and not added)
    for (uint32_t s = 0; s < p.parts; s += AT_ONCE) {
        floatx4 lo[AT_ONCE], hi[AT_ONCE];
#pragma unroll
        for (uint32_t i = 0; i < AT_ONCE; ++i) {
            const float* at = from + (s + i < p.parts ? s + i : p.parts - 1u) * apart;
            lo[i] = reinterpret_cast<const floatx4*>(at)[0];
            hi[i] = reinterpret_cast<const floatx4*>(at)[1];
        }
#pragma unroll
        for (uint32_t i = 0; i < AT_ONCE; ++i)
#pragma unroll
            for (uint32_t n = 0; n < 4u; ++n) {
                h[n] += s + i < p.parts ? lo[i][n] : 0.0f;
                h[n + 4u] += s + i < p.parts ? hi[i][n] : 0.0f;
            }
    }
}
// Block `block` of a row's terms, [term][block][8] behind `to`, from these ranks; `adapted`: the row has an adapter.  A term is the upper half of what is left of h: 8 of its 24
// bits (and of an infinity or a NaN all that it says; nothing is left of these).
__device__ __forceinline__ void write_terms(const AdaptParams& p, bool adapted, uint32_t block, float (&h)[8], uint16_t* to) {
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) h[i] = __builtin_canonicalizef(adapted && block < p.blocks && block * 8u + i < p.rank ? h[i] : 0.0f);
#pragma unroll
    for (uint32_t term = 0; term < kTerms; ++term) {
        if (term && block >= p.blocks) break;
        words4 w;
#pragma unroll
        for (uint32_t i = 0; i < 8u; i += 2u) w[i >> 1] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, h[i + 1u]), __builtin_bit_cast(uint32_t, h[i]), 0x07060302u);
        *reinterpret_cast<words4*>(to + (term * p.blocks + block) * 8u) = w;
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) {
            const float left = h[i] - bf16_high(__builtin_bit_cast(uint32_t, h[i]));
            h[i] = term || __builtin_fabsf(h[i]) < __builtin_inff() ? left : 0.0f;
        }
    }
}
// Which blocks there are to write: each of the first term, which writes the others too, and those behind all terms, which are zeros.
__device__ __forceinline__ bool writes(const AdaptParams& p, uint32_t block) { return block < p.blocks || block >= p.blocks * kTerms; }

// 8 consecutive elements of an operand that has as many in a row.
template <uint32_t DTYPE>
__device__ __forceinline__ Eight<DTYPE> eight(const void* base, uint64_t at) {
    Eight<DTYPE> to;
    const uint8_t* const from = static_cast<const uint8_t*>(base) + at * (DTYPE == ANSZP_OUT_BF16 ? 2u : 4u);
    if constexpr (DTYPE == ANSZP_OUT_BF16) {
        to.w = *reinterpret_cast<const words4_any*>(from);
    } else {
        to.w[0] = *reinterpret_cast<const words4_any*>(from);
        to.w[1] = *reinterpret_cast<const words4_any*>(from + 16);
    }
    return to;
}
// The 8 columns that a lane with the ones from `col` on works at: where fewer are left the last 8 of the row, of which it stores its own.
struct Eighth {
    uint64_t at;
    uint32_t skip;                      // columns that are another lane's, 8: all are
    __device__ __forceinline__ Eighth(uint64_t col, uint64_t cols) : at(least(col, cols - 8u)), skip(col < cols ? uint32_t(col - at) : 8u) {}
};
template <uint32_t BASE, uint32_t OUT>
__device__ __forceinline__ void finish(const AdaptParams& p, uint64_t row, const Eighth& cols, const Eight<BASE>& base, const Eight<OUT>& beside, bool adds, const float (&sum)[8]) {
    float v[8];
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) v[i] = adds ? base[i] + sum[i] : base[i];
    const auto each = [&](uint32_t activation) __attribute__((always_inline)) {
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) v[i] = activated(v[i], activation);
    };
    switch (p.activation) {                                         // (once for the eight, not for each)
        case ANSZP_FN_RELU: each(ANSZP_FN_RELU); break;
        case ANSZP_FN_GELU: each(ANSZP_FN_GELU); break;
        case ANSZP_FN_SILU: each(ANSZP_FN_SILU); break;
        default: break;
    }
    if (p.mul) {
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) v[i] *= beside[i];
    }
    if (p.residual) {
        if (p.mul) {
            const Eight<OUT> residual = eight<OUT>(p.residual, row * p.residual_stride + cols.at);
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) v[i] += residual[i];
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) v[i] += beside[i];
        }
    }
    const uint64_t at = row * p.out_stride + cols.at;
    if (cols.skip == 0u) {
        store_eight(p.out, OUT, at, 8u, v);
        return;
    }
#pragma unroll
    for (uint32_t i = 1; i < 8u; ++i) {
        if (i < cols.skip) continue;
        if constexpr (OUT == ANSZP_OUT_BF16) static_cast<uint16_t*>(p.out)[at + i] = to_bf16(v[i]);
        else static_cast<float*>(p.out)[at + i] = v[i];
    }
}
// Eight ranks of a row of b: block `block` of it.
template <bool WHOLE>
__device__ __forceinline__ words4 ranks_of(const AdaptParams& p, const uint16_t* row, uint32_t block) {
    const uint8_t* const at = reinterpret_cast<const uint8_t*>(row + block * 8u);
    if constexpr (WHOLE) return *reinterpret_cast<const words4_any*>(at);
    else return careful(at, 2 * (int32_t(p.rank) - int32_t(block) * 8), p.b_last);
}
// Steps of the second product, each of four blocks of a row of b, which meet h's terms one after the other.  Of one or two blocks the four are the same again: they meet
// several terms at once.
struct Steps {
    uint32_t steps, turns, apart;       // turns of a step, and how far apart what they take of h lies
    __device__ __forceinline__ explicit Steps(const AdaptParams& p)
        : steps(p.blocks < 4u ? 1u : p.blocks / 4u), turns(p.blocks < 4u ? p.width / 32u : kTerms), apart(p.blocks < 4u ? 32u : p.blocks * 8u) {}
};
__device__ __forceinline__ uint32_t block_of(const AdaptParams& p, uint32_t step, uint32_t g) { return p.blocks < 4u ? g & (p.blocks - 1u) : step * 4u + g; }

// The ids of a tile's rows, one a lane; rows that are not there have the last one's.
__device__ __forceinline__ int32_t tile_ids(const AdaptParams& p, uint64_t first, bool tells) {
    const uint64_t row = first + (threadIdx.x & 63u);
    return id_of(p, least(row, p.rows - 1u), tells && row < p.rows);
}

// The parts of k added up and h's terms, [row][term][block][8] with zeros where there is none, for many rows; a block a thread.
__global__ __launch_bounds__(256) void adapt_terms_kernel(AdaptParams p) {
    const uint32_t room = p.width / 8u;
    const uint64_t n = uint64_t(blockIdx.x) * 256u + threadIdx.x, row = n / room;
    const uint32_t block = uint32_t(n - row * room);
    if (row >= p.rows || !writes(p, block)) return;
    float h[8] = {};
    if (block * 8u < p.rank && block < p.blocks) {
        if (p.parts > 4u) load_h<16u>(p, row, block, h);
        else load_h<4u>(p, row, block, h);
    }
    write_terms(p, uint32_t(p.ids[row]) < p.adapters, block, h, p.terms_of_h + row * p.width);
}

// Many rows: 16 of them and 128 columns a wavefront, 64 of them a workgroup, which has b's rows of its columns in LDS.  In the instructions' terms h's rows are the rows and
// every eighth of b's a column, so that a lane ends up with 8 consecutive columns of four rows and 16 lanes with a row's 128: operands and results move 256
// bytes of a row (of bf16) at a time.
template <uint32_t BASE, uint32_t OUT, bool WHOLE>
__global__ __launch_bounds__(256, BASE == ANSZP_OUT_BF16 && OUT == ANSZP_OUT_BF16 ? 4 : 3) void adapt_up_kernel(AdaptParams p) {
    extern __shared__ __attribute__((aligned(16))) uint16_t b_rows[];                              // [column / 8 in steps of 8][block][8], 8 more behind a row
    const uint32_t lane = threadIdx.x & 63u, c = lane & 15u, g = lane >> 4, wave = threadIdx.x >> 6;
    const uint32_t tile = blockIdx.x / p.across, piece = blockIdx.x - tile * p.across;
    const uint64_t top = uint64_t(tile) * 64u, first = least(top + wave * 16u, p.rows - 1u);
    const int32_t id = tile_ids(p, top, piece == 0u && wave == 0u);
    const Eighth cols(uint64_t(piece) * 128u + c * 8u, p.cols);
    const uint32_t rows = uint32_t(least(p.rows - top, 64u)), width = p.blocks * 8u + 8u;
    const Steps of(p);
    const uint16_t* const h_at = p.terms_of_h + least(first + c, p.rows - 1u) * p.width + g * 8u;
    uint64_t left = ~0ull >> (64u - rows);
    bool staged = false;
    while (left) {
        const int32_t one = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        const uint64_t same = __ballot(id == one) & left;
        const uint32_t mine = uint32_t(same >> (wave * 16u)) & 0xFFFFu;
        left &= ~same;
        // (a turn works out its addresses itself: the compiler would do it once, for the turns that hardly ever come, and keep 40 registers for them)
        uint32_t row_of = wave * 16u + 4u * g, thread = threadIdx.x;
        asm volatile("" : "+v"(row_of), "+v"(thread));
        // (out may be one of the operands, so what a row has is asked for before anything of it is stored)
        Eight<BASE> base[4];
        Eight<OUT> beside[4];
        if (mine) {
#pragma unroll
            for (uint32_t i = 0; i < 4u; ++i) {
                const uint64_t row = least(top + row_of + i, p.rows - 1u);
                base[i] = eight<BASE>(p.base, row * p.base_stride + cols.at);
                if (p.mul) beside[i] = eight<OUT>(p.mul, row * p.mul_stride + cols.at);
                else if (p.residual) beside[i] = eight<OUT>(p.residual, row * p.residual_stride + cols.at);
            }
        }
        floatx4 sum[8] = {};
        if (one >= 0) {
            if (staged) __syncthreads();
            staged = true;
            const uint16_t* const b = p.b + uint64_t(one) * p.b_stride;
            for (uint32_t n = thread; n < 128u * p.blocks; n += 1024u) {
                words4 w[4];
#pragma unroll
                for (uint32_t i = 0; i < 4u; ++i) {
                    const uint32_t at = n + i * 256u, j = at / p.blocks, block = at - j * p.blocks;
                    if (at < 128u * p.blocks) w[i] = ranks_of<WHOLE>(p, b + (least(uint64_t(piece) * 128u + (j & ~7u), p.cols - 8u) + (j & 7u)) * p.b_row_stride, block);
                }
#pragma unroll
                for (uint32_t i = 0; i < 4u; ++i) {
                    const uint32_t at = n + i * 256u, j = at / p.blocks, block = at - j * p.blocks;
                    if (at < 128u * p.blocks) *reinterpret_cast<words4*>(b_rows + ((j & 7u) * 16u + (j >> 3)) * width + block * 8u) = w[i];
                }
            }
            __syncthreads();
            if (mine) {
                // (a step's terms are under way together, 161 us a call of 8192 rows; one after the other 171)
#pragma unroll 1
                for (uint32_t s = 0; s < of.steps; ++s) {
                    words4 h[kTerms];
#pragma unroll
                    for (uint32_t u = 0; u < kTerms; ++u) h[u] = *reinterpret_cast<const words4*>(h_at + s * 32u + (u < of.turns ? u : 0u) * of.apart);
                    const uint16_t* const b_at = b_rows + c * width + block_of(p, s, g) * 8u;
#pragma unroll
                    for (uint32_t t = 0; t < 8u; ++t) {
                        const bf16x8 b = *reinterpret_cast<const bf16x8*>(b_at + t * 16u * width);
#pragma unroll
                        for (uint32_t u = 0; u < kTerms; ++u)
                            if (u < of.turns) sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(h[u]), b, sum[t], 0, 0, 0);
                    }
                }
            }
        }
        if (!mine || cols.skip == 8u) continue;
#pragma unroll
        for (uint32_t i = 0; i < 4u; ++i) {
            if (!(mine >> (4u * g + i) & 1u)) continue;
            const float v[8] = {sum[0][i], sum[1][i], sum[2][i], sum[3][i], sum[4][i], sum[5][i], sum[6][i], sum[7][i]};
            finish<BASE, OUT>(p, top + row_of + i, cols, base[i], beside[i], one >= 0, v);
        }
    }
}

// Few rows: 64 of them and 32 columns a workgroup, whose wavefronts have every fourth of the rows' adapters, with the rows they are of.  In the instructions'
// terms b's rows are the rows, in an order that leaves each lane with 8 consecutive columns of its row.  Four pieces of adapters are under way, so that a wavefront
// waits for memory once, not for each.
template <uint32_t BASE, uint32_t OUT, bool WHOLE>
__global__ __launch_bounds__(256, 2) void adapt_up_few_kernel(AdaptParams p) {
    constexpr uint32_t kRing = 4u;
    extern __shared__ __attribute__((aligned(16))) uint16_t terms_of_h[];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, c = lane & 15u, g = lane >> 4;
    const uint32_t tile = blockIdx.x / p.across, piece = blockIdx.x - tile * p.across;
    const uint64_t first = uint64_t(tile) * 64u;
    const Eighth cols(uint64_t(piece) * 32u + g * 8u, p.cols), cols_of_b(uint64_t(piece) * 32u + (c >> 2) * 8u, p.cols);
    // All that does not wait for the rows' ids is asked for first: their operands, and the first piece of h that this thread writes to LDS.
    Eight<BASE> base[4];
    Eight<OUT> beside[4];
#pragma unroll
    for (uint32_t r = 0; r < 4u; ++r) {
        const uint64_t row = least(first + r * 16u + c, p.rows - 1u);
        base[r] = eight<BASE>(p.base, row * p.base_stride + cols.at);
        if (p.mul) beside[r] = eight<OUT>(p.mul, row * p.mul_stride + cols.at);
        else if (p.residual) beside[r] = eight<OUT>(p.residual, row * p.residual_stride + cols.at);
    }
    float h[8] = {};
    if (wave < p.blocks && wave * 8u < p.rank) load_h<4u>(p, least(first + lane, p.rows - 1u), wave, h);
    const int32_t id = tile_ids(p, first, piece == 0u && wave == 0u);
    const uint32_t of_wave = (id < 0 ? lane : uint32_t(id) ^ uint32_t(id) >> 2 ^ uint32_t(id) >> 4) & 3u;          // (rows without an adapter are anyone's)
    // A piece of an adapter: four blocks of its ranks.
    struct Piece {
        words4 b[2];
        int32_t one;
        uint32_t s;
        uint64_t lanes;
    } ring[kRing];
    const Steps of(p);
    const uint16_t* const b_at = p.b + (cols_of_b.at + (c & 3u)) * p.b_row_stride;
    Adapters adapters(of_wave == wave ? id : -1);
    int32_t asked = -1;
    uint32_t asked_at = of.steps;
    const auto ask = [&](Piece& to) __attribute__((always_inline)) {
        if (++asked_at >= of.steps) {
            asked = adapters.next();
            asked_at = 0u;
        }
        to.one = asked;
        to.s = asked_at;
        to.lanes = adapters.lanes;
        if (asked < 0) return;
#pragma unroll
        for (uint32_t t = 0; t < 2u; ++t) to.b[t] = ranks_of<WHOLE>(p, b_at + uint64_t(asked) * p.b_stride + t * 4u * p.b_row_stride, block_of(p, asked_at, g));
    };
#pragma unroll
    for (uint32_t i = 0; i < kRing; ++i) ask(ring[i]);
    int32_t own[4];
    bool mine[4];
#pragma unroll
    for (uint32_t r = 0; r < 4u; ++r) {
        own[r] = __shfl(id, r * 16u + c);
        mine[r] = __shfl(of_wave, r * 16u + c) == wave && first + r * 16u + c < p.rows;
    }
    for (uint32_t block = wave; block < p.width / 8u; block += 4u) {
        if (!writes(p, block)) continue;
        if (block != wave && block < p.blocks && block * 8u < p.rank) load_h<4u>(p, least(first + lane, p.rows - 1u), block, h);
        write_terms(p, id >= 0, block, h, terms_of_h + lane * (p.width + 8u));
    }
    // (out may be one of the operands: what another wavefront stores has been read by all behind this, too)
    __syncthreads();
    const uint16_t* const h_at = terms_of_h + c * (p.width + 8u) + g * 8u;
    floatx4 sum[4][2] = {}, part[4][2] = {};
    for (bool more = true; more;) {
#pragma unroll
        for (uint32_t i = 0; i < kRing; ++i) {
            Piece& now = ring[i];
            if (now.one < 0) {
                more = false;
                break;
            }
#pragma unroll
            for (uint32_t r = 0; r < 4u; ++r) {
                if (!(now.lanes >> (16u * r) & 0xFFFFu)) continue;
                const auto multiply = [&](uint32_t turn) __attribute__((always_inline)) {
                    const bf16x8 h = *reinterpret_cast<const bf16x8*>(h_at + r * 16u * (p.width + 8u) + now.s * 32u + turn * of.apart);
#pragma unroll
                    for (uint32_t t = 0; t < 2u; ++t) part[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(now.b[t]), h, part[r][t], 0, 0, 0);
                };
#pragma unroll
                for (uint32_t u = 0; u < kTerms; ++u)
                    if (u < of.turns) multiply(u);
            }
            if (now.s + 1u == of.steps) {
#pragma unroll
                for (uint32_t r = 0; r < 4u; ++r) {
                    if (!(now.lanes >> (16u * r) & 0xFFFFu)) continue;
#pragma unroll
                    for (uint32_t t = 0; t < 2u; ++t) {
                        sum[r][t] = own[r] == now.one ? part[r][t] : sum[r][t];
                        part[r][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
                    }
                }
            }
            ask(now);
        }
    }
    if (cols.skip == 8u) return;
#pragma unroll
    for (uint32_t r = 0; r < 4u; ++r) {
        if (!mine[r]) continue;
        const float v[8] = {sum[r][0][0], sum[r][0][1], sum[r][0][2], sum[r][0][3], sum[r][1][0], sum[r][1][1], sum[r][1][2], sum[r][1][3]};
        finish<BASE, OUT>(p, first + r * 16u + c, cols, base[r], beside[r], own[r] >= 0, v);
    }
}

// Operands of fewer than 16 bytes, and rows of fewer than 8 columns: an element a thread.
template <bool BYTES>
__global__ __launch_bounds__(256) void adapt_down_any_kernel(AdaptParams p) {
    const uint64_t n = uint64_t(blockIdx.x) * 256u + threadIdx.x, row = n / p.rank;
    const uint32_t rank = uint32_t(n - row * p.rank);
    if (row >= p.rows) return;
    const int32_t one = id_of(p, row, false);
    if (one < 0) return;
    float sum = 0.0f;
    for (uint32_t i = 0; i < p.k; ++i) {
        const uint8_t* const x = p.x + row * p.x_stride;
        const float v = BYTES ? float(reinterpret_cast<const int8_t*>(x)[i]) : bf16_low(reinterpret_cast<const uint16_t*>(x)[i]);
        sum = fmaf(v, bf16_low(p.a[uint64_t(one) * p.a_stride + rank * p.a_row_stride + i]), sum);
    }
    p.h[row * p.rank_room + rank] = (p.scales ? p.scales[one] : 1.0f) * (p.x_scales ? p.x_scales[row] : 1.0f) * sum;
}
template <uint32_t BASE, uint32_t OUT>
__global__ __launch_bounds__(256) void adapt_up_any_kernel(AdaptParams p) {
    const uint64_t n = uint64_t(blockIdx.x) * 256u + threadIdx.x, row = n / p.cols, col = n - row * p.cols;
    if (row >= p.rows) return;
    const int32_t one = id_of(p, row, col == 0u);
    const auto value = [](const void* at, uint32_t dtype, uint64_t i) __attribute__((always_inline)) {
        return dtype == ANSZP_OUT_BF16 ? bf16_low(static_cast<const uint16_t*>(at)[i]) : static_cast<const float*>(at)[i];
    };
    float v = 0.0f;
    if (one >= 0)
        for (uint32_t i = 0; i < p.rank; ++i) {
            float h = 0.0f;
            for (uint32_t s = 0; s < p.parts; ++s) h += p.h[(s * p.rows + row) * p.rank_room + i];
            v = fmaf(h, bf16_low(p.b[uint64_t(one) * p.b_stride + col * p.b_row_stride + i]), v);
        }
    const float base = value(p.base, BASE, row * p.base_stride + col);
    v = activated(one >= 0 ? base + v : base, p.activation);
    if (p.mul) v *= value(p.mul, OUT, row * p.mul_stride + col);
    if (p.residual) v += value(p.residual, OUT, row * p.residual_stride + col);
    if constexpr (OUT == ANSZP_OUT_BF16) static_cast<uint16_t*>(p.out)[row * p.out_stride + col] = to_bf16(v);
    else static_cast<float*>(p.out)[row * p.out_stride + col] = v;
}

struct Plan {
    uint32_t ranks;                     // 16s of ranks a workgroup of the first product has
    uint32_t slots, groups, parts, blocks, width;
    bool few, any_down, any_up;         // few rows; operands too short for the kernels of tiles
    uint64_t sums, workspace;           // bytes of the sums of k's parts, of all
};

int adapt_check(const anszp_adapt_args_t& a) {
    if ((a.x_dtype != ANSZP_OUT_BF16 && a.x_dtype != ANSZP_I8) || (a.base_dtype != ANSZP_OUT_F32 && a.base_dtype != ANSZP_OUT_BF16) ||
        (a.out_dtype != ANSZP_OUT_F32 && a.out_dtype != ANSZP_OUT_BF16) || a.activation > ANSZP_FN_SILU || a.k == 0 || a.k > 1u << 30 || a.rank == 0 || a.rank > 128u ||
        a.rows >= 1ull << 28 || a.cols >= 1ull << 31 || a.adapters >= 1u << 24)
        return ANSZP_E_RANGE;
    if (a.rows > 1 && a.out_stride < a.cols) return ANSZP_E_RANGE;
    return ANSZP_OK;
}

// Bytes from an operand's first element to its last.
uint64_t bytes_of_x(const anszp_adapt_args_t& a) { return ((a.rows > 1 ? (a.rows - 1u) * a.x_stride : 0u) + a.k) * (a.x_dtype == ANSZP_I8 ? 1u : 2u); }
uint64_t bytes_of(const anszp_adapt_args_t& a, uint64_t stride, uint64_t rows, uint64_t row_stride, uint64_t width) {
    return a.adapters ? ((a.adapters > 1u ? (a.adapters - 1ull) * stride : 0u) + (rows > 1u ? (rows - 1u) * row_stride : 0u) + width) * 2u : 0u;
}

Plan plan_of(const anszp_adapt_args_t& a) {
    Plan q = {};
    if (a.adapters == 0u) {
        q.blocks = 1u;
        q.width = 32u;
        return q;
    }
    const uint32_t tiles = static_cast<uint32_t>((a.rows + 63u) / 64u), sixteens = (a.rank + 15u) / 16u;
    q.ranks = sixteens <= 1u ? 1u : sixteens <= 2u ? 2u : 4u;
    const uint32_t once = at_once(a.x_dtype == ANSZP_I8, q.ranks), steps = (a.k + once - 1u) / once;
    q.groups = (sixteens + q.ranks - 1u) / q.ranks;
    // A step's rows may have an adapter each, a prompt's tiles have one or two: workgroups whose rows are not the first of an adapter leave at once.  (1531
    // rows with five adapters 15.3 us with two workgroups that share a tile's adapters, 18.8 with five: each asks for its tile's ids before it can leave.)
    // k in parts until there are two workgroups a CU.  Where a workgroup of the second product adds them up for 64 rows itself, with hundreds of such workgroups, parts have
    // eight steps at least (256 rows to 11008 with four adapters, k of 4096: four parts 26.6 us, sixteen 28.7; k of 11008 to 4096: four 26.7, ten 19.4).
    const uint32_t rows = static_cast<uint32_t>(a.rows < 64u ? a.rows : 64u), likely = a.rows < 512u ? (rows < a.adapters ? rows : a.adapters) : 1u;
    q.slots = a.rows < 512u ? rows : a.adapters < 2u ? 1u : a.adapters <= 8u || a.rows >= 4096u ? 2u : 8u;
    const uint32_t groups = tiles * likely * q.groups, most = (steps + 1u) / 2u, read_again = a.rows <= 64u || a.rows > 256u || steps > 128u ? 16u : steps > 32u ? steps / 8u : 4u;
    q.parts = (2u * device_cus() + groups - 1u) / groups;
    if (q.parts > read_again) q.parts = read_again;
    if (q.parts > most) q.parts = most;
    q.any_down = bytes_of_x(a) < 16u || bytes_of(a, a.a_stride, a.rank, a.a_row_stride, a.k) < 16u;
    q.any_up = a.cols < 8u || bytes_of(a, a.b_stride, a.cols, a.b_row_stride, a.rank) < 16u;
    if (q.any_down) q.parts = 1u;
    const uint32_t blocks = (a.rank + 7u) / 8u;
    // Few rows: adapters at the same time, in a kernel that reads all of h for 32 columns and has no terms' kernel before it.  (64 rows to 11008: one
    // adapter 13.7 us, else 14.7; four, mixed, 14.1 to 21.5; 256 rows: 16, mixed, 34 to 46; two, 128 rows each, 26.7 to 18; four, 64 each, 26.6 to 18.  512:
    // eight, 64 each, 43 to 16; 48, mixed, 88 to 100.)
    q.few = q.any_up || a.rows <= 64u || (a.rows <= 256u && a.adapters >= 4u);
    q.blocks = blocks <= 2u ? blocks : (blocks + 3u) / 4u * 4u;     // (a step of the second product has four blocks: of one term, or of several short ones)
    q.width = (q.blocks * kTerms + 3u) / 4u * 32u;
    q.sums = (q.parts * a.rows * blocks * 32u + 15u) & ~15ull;
    q.workspace = q.sums + (q.few ? 0u : a.rows * q.width * 2u);
    return q;
}

template <bool BYTES>
void launch_down(const AdaptParams& p, const Plan& q, hipStream_t s) {
    if (q.any_down) {
        hipLaunchKernelGGL(adapt_down_any_kernel<BYTES>, dim3(static_cast<uint32_t>((p.rows * p.rank + 255u) / 256u)), dim3(256), 0, s, p);
        return;
    }
    const dim3 grid(static_cast<uint32_t>((p.rows + 63u) / 64u), q.slots * q.groups, q.parts), threads(256);
    if (q.ranks == 1u) hipLaunchKernelGGL((adapt_down_kernel<BYTES, 1u>), grid, threads, 0, s, p);
    else if (q.ranks == 2u) hipLaunchKernelGGL((adapt_down_kernel<BYTES, 2u>), grid, threads, 0, s, p);
    else hipLaunchKernelGGL((adapt_down_kernel<BYTES, 4u>), grid, threads, 0, s, p);
}

template <uint32_t BASE, uint32_t OUT, bool WHOLE>
void launch_up(AdaptParams& p, bool few, hipStream_t s) {
    const uint32_t tiles = static_cast<uint32_t>((p.rows + 63u) / 64u);
    p.across = static_cast<uint32_t>(few ? (p.cols + 31u) / 32u : (p.cols + 127u) / 128u);
    if (few) hipLaunchKernelGGL((adapt_up_few_kernel<BASE, OUT, WHOLE>), dim3(p.across * tiles), dim3(256), 64u * (p.width + 8u) * 2u, s, p);
    else hipLaunchKernelGGL((adapt_up_kernel<BASE, OUT, WHOLE>), dim3(p.across * tiles), dim3(256), 128u * (p.blocks * 8u + 8u) * 2u, s, p);
}
template <uint32_t BASE, uint32_t OUT>
void launch_up(AdaptParams& p, bool any, bool few, hipStream_t s) {
    if (any) hipLaunchKernelGGL((adapt_up_any_kernel<BASE, OUT>), dim3(static_cast<uint32_t>((p.rows * p.cols + 255u) / 256u)), dim3(256), 0, s, p);
    else if (p.rank % (p.blocks < 4u ? 8u : 32u) == 0u) launch_up<BASE, OUT, true>(p, few, s);          // (no block of ranks ends early)
    else launch_up<BASE, OUT, false>(p, few, s);
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
    if (meet(out, {a->x_scales, 1, 0, a->rows * 4u}) || meet(out, {a->scales, 1, 0, a->adapters * 4u}) || meet(out, {a->x, a->rows, a->x_stride * x_size, a->k * x_size}) ||
        meet(out, {a->ids, 1, 0, a->rows * 4u}) ||
        (base_size == size ? meet_elsewhere(out, base) : meet(out, base)) || meet_elsewhere(out, {a->mul, a->rows, a->mul_stride * size, width}) ||
        meet_elsewhere(out, {a->residual, a->rows, a->residual_stride * size, width}) ||
        meet(out, {a->a, 1, 0, ((a->adapters - 1ull) * a->a_stride + (a->rank - 1ull) * a->a_row_stride + a->k) * (a->adapters ? 2u : 0u)}) ||
        meet(out, {a->b, 1, 0, ((a->adapters - 1ull) * a->b_stride + (a->cols - 1ull) * a->b_row_stride + a->rank) * (a->adapters ? 2u : 0u)}))
        return ANSZP_E_RANGE;
    if ((a->rows + 63u) / 64u * ((a->cols + 31u) / 32u) >= 1ull << 24) return ANSZP_E_RANGE;          // (threads that one launch has not)
    const Plan q = plan_of(*a);
    constexpr uint64_t kMost = (1ull << 32) - 256u;                 // threads that launches an element a thread have, in workgroups of 256
    const bool any = q.any_up || a->cols < 8u;                      // (also where there are no adapters)
    if (a->rows * (q.width / 8u) > kMost || (q.any_down && a->rows * a->rank > kMost) || (any && a->rows * a->cols > kMost)) return ANSZP_E_RANGE;
    if (q.workspace && !a->workspace) return ANSZP_E_NULL;
    if (q.workspace && (a->workspace_bytes < q.workspace || (reinterpret_cast<uintptr_t>(a->workspace) & 15u))) return ANSZP_E_RANGE;
    AdaptParams p = {};
    p.x = static_cast<const uint8_t*>(a->x); p.a = static_cast<const uint16_t*>(a->a); p.b = static_cast<const uint16_t*>(a->b);
    p.ids = a->ids; p.x_scales = a->x_scales; p.scales = a->scales; p.base = a->base; p.mul = a->mul; p.residual = a->residual; p.out = a->out;
    p.h = static_cast<float*>(a->workspace); p.status = a->status;
    p.x_stride = a->x_stride * x_size; p.a_stride = a->a_stride; p.a_row_stride = a->a_row_stride; p.b_stride = a->b_stride; p.b_row_stride = a->b_row_stride;
    p.base_stride = a->base_stride; p.mul_stride = a->mul_stride; p.residual_stride = a->residual_stride; p.out_stride = a->out_stride;
    p.rows = a->rows; p.cols = a->cols; p.adapters = a->adapters; p.k = a->k; p.rank = a->rank; p.rank_room = (a->rank + 7u) / 8u * 8u;
    p.activation = a->activation;
    p.slots = q.slots; p.groups = q.groups; p.parts = q.parts;
    p.blocks = q.blocks; p.width = q.width;
    p.x_last = p.x + bytes_of_x(*a) - 16u;
    p.a_last = reinterpret_cast<const uint8_t*>(p.a) + bytes_of(*a, a->a_stride, a->rank, a->a_row_stride, a->k) - 16u;
    p.b_last = reinterpret_cast<const uint8_t*>(p.b) + bytes_of(*a, a->b_stride, a->cols, a->b_row_stride, a->rank) - 16u;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (q.workspace) {
        p.terms_of_h = reinterpret_cast<uint16_t*>(static_cast<uint8_t*>(a->workspace) + q.sums);
        if (bytes) launch_down<true>(p, q, s);
        else launch_down<false>(p, q, s);
        if (!q.few) hipLaunchKernelGGL(adapt_terms_kernel, dim3(static_cast<uint32_t>((a->rows * (q.width / 8u) + 255u) / 256u)), dim3(256), 0, s, p);
    }
    const bool base_short = a->base_dtype == ANSZP_OUT_BF16, out_short = a->out_dtype == ANSZP_OUT_BF16;
    if (base_short && out_short) launch_up<ANSZP_OUT_BF16, ANSZP_OUT_BF16>(p, any, q.few, s);
    else if (base_short) launch_up<ANSZP_OUT_BF16, ANSZP_OUT_F32>(p, any, q.few, s);
    else if (out_short) launch_up<ANSZP_OUT_F32, ANSZP_OUT_BF16>(p, any, q.few, s);
    else launch_up<ANSZP_OUT_F32, ANSZP_OUT_F32>(p, any, q.few, s);
    return hipGetLastError() == hipSuccess ? ANSZP_OK : ANSZP_E_HIP;
}
