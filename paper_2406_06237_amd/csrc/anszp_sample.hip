// The next token of each row drawn from its logits, for gfx950.  With l the logits, tokens in the order of falling l (equal ones: the lower first) and
//   w = exp((l - max l) / temperature)
// a row keeps the shortest of these beginnings of the order: the first top_k; of those the shortest whose weights reach top_p of theirs; the ones with
// w >= min_p.  It draws the first token at which the sum of the kept weights passes uniform * (their sum).
//
// Sums decide which token it is, so they are whole numbers and no order of additions changes them.  With t = 64 log2(e) (max l - l) / temperature, in 64
// bits, and b = round(t):
//   w = 2^(-b / 64) * q,    q = 2^((b - t) / 64) in 1 +- 0.0054, which a polynomial of three powers gives to 5e-12,
// the q are held in fixed point with 2^-44 (less only for more than 2^18 tokens) and added up for each b in LDS; a bin's mass is its sum times
// 2^(-b / 64), rounded down, and masses are added up over the bins.  What is further down than 44 octaves weighs nothing.  Weights of 32 bits would not do: of 10000
// tokens that are kept, one in 100000 draws would be another token than the formula's.  The bins say in which of them the border and the token are; the tokens of these are
// listed, a few hundred, and each is compared with all others.  Where they are more than the list holds, each bin is cut by its tokens' own logits, as often
// as that takes.  A small top_k needs no bins: a list of all tokens that may be kept is found by the threads' own largest.
//
// Instructions bound it, not memory: 512 rows of 131072 in bf16 take 87 us, 1.5 TB/s, 30 instructions of the vector unit a logit, about half of them for q, with
// the unit busy 58 % of the time and LDS 28 (an addition to a bin of each of 64 lanes takes 14 clocks, 8 of them for banks that meet).  One row of 32000
// takes 15 us: each of three passes waits for its first loads, and the sums between them for each other.
#include <hip/hip_runtime.h>

#include "anszp_cus.h"
#include "anszp_numbers.h"

namespace {

constexpr uint32_t kSteps = 64, kBins = 44u * kSteps, kList = 512, kCuts = 512;

struct SampleParams {
    const void* logits;
    const float* uniforms;
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    int64_t* tokens;
    float* chances;
    uint64_t rows, stride;
    uint32_t vocabulary;
    int32_t any_top_k;
    float any_temperature, any_top_p, any_min_p;
    uint32_t point;                     // binary digits behind the point of q and of masses
};

// Logits in the order of their numbers; both zeros are one.
__device__ __forceinline__ uint32_t key_of(float l) {
    const uint32_t w = __builtin_bit_cast(uint32_t, l + 0.0f);
    return w ^ (w >> 31 ? ~0u : 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t key) { return __builtin_bit_cast(float, key ^ (key >> 31 ? 0x80000000u : ~0u)); }

// A token in a list: `order` is larger the earlier it comes.
struct Entry {
    uint64_t order, q;                  // (its q, or its mass)
};
__device__ __forceinline__ uint64_t order_of(uint32_t key, uint32_t id) { return uint64_t(key) << 32 | ~id; }
__device__ __forceinline__ uint32_t id_of(const Entry& e) { return ~uint32_t(e.order); }

struct Shared {
    Entry list[kList];
    uint64_t mass[kBins + 1u];          // first the sums of q, then the masses before each bin
    uint64_t cut_sum[kCuts];
    double octave[kSteps];              // 2^(-i / 64)
    uint64_t of_wave[16], of_wave_too[16];
    uint32_t count[kBins + 1u];         // first the tokens, then those before each bin
    uint32_t cut_count[kCuts];
    uint32_t list_bin[kList];
    uint32_t listed, least, most;
    uint32_t found, found_too, found_id;
    uint32_t found_top_p;               // (a word of its own: what marks the next bin waits for no one who still reads this one)
    uint64_t found_sum, found_q, found_count;
};

__device__ __forceinline__ double height(const Shared& sh, uint32_t bin) { return ldexp(sh.octave[bin % kSteps], -int(bin / kSteps)); }
__device__ __forceinline__ uint64_t mass_of(double height, uint64_t sum) { return uint64_t(height * double(sum)); }

// The largest of `v` over a wavefront.  (Lanes trade by their place in a row of 16 as operands, without LDS.)
template <int CONTROL>
__device__ __forceinline__ uint32_t traded(uint32_t v) {
    return uint32_t(__builtin_amdgcn_mov_dpp(int(v), CONTROL, 0xF, 0xF, true));
}
__device__ __forceinline__ uint32_t most_of_wave(uint32_t v) {
    const auto with = [&](uint32_t other) __attribute__((always_inline)) { v = other > v ? other : v; };
    with(traded<0xB1>(v));                                          // quad_perm [1, 0, 3, 2]
    with(traded<0x4E>(v));                                          // quad_perm [2, 3, 0, 1]
    with(traded<0x141>(v));                                         // a half row mirrored
    with(traded<0x140>(v));                                         // a row mirrored
    with(__shfl_xor(v, 16));
    with(__shfl_xor(v, 32));
    return v;
}

// A row and the workgroup of THREADS threads that has it, which reads it for each pass.  (Rows up to 32768 held in registers, 64 of them a thread, took as
// long where rows are few and half as long again where they are many, 512 of 20000 30 us instead of 20: one workgroup a CU has the registers.)
template <uint32_t DTYPE, uint32_t THREADS>
struct Row {
    static constexpr uint32_t kWaves = THREADS / 64u;
    Shared& sh;
    const void* logits;
    uint64_t from;
    uint32_t n, point;
    double top, steps, shift;           // the largest logit, 64 log2(e) / temperature, their product
    double c0, c1, c2, c3, one;         // of q
    bool far;

    // Eight logits, in pieces of 16 bytes so that the lanes of a load lie next to each other: of fp32 four, and four a workgroup's load further.
    // Behind the row's end there is nothing that weighs.
    static constexpr uint32_t kPiece = DTYPE == ANSZP_OUT_BF16 ? 8u : 4u, kApart = THREADS * kPiece;
    static __device__ __forceinline__ uint32_t token_of(uint32_t at, uint32_t i) { return at + i / kPiece * kApart + i % kPiece; }
    __device__ __forceinline__ Eight<DTYPE> eight(uint32_t at) const {
        Eight<DTYPE> l;
        if constexpr (DTYPE == ANSZP_OUT_BF16) {
            l.w = *reinterpret_cast<const words4_any*>(static_cast<const uint16_t*>(logits) + from + at);
        } else {
#pragma unroll
            for (uint32_t j = 0; j < 2u; ++j) l.w[j] = *reinterpret_cast<const words4_any*>(static_cast<const float*>(logits) + from + at + j * kApart);
        }
        return l;
    }
    __device__ __forceinline__ Eight<DTYPE> last_eight(uint32_t at) const {
        Eight<DTYPE> l;
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) {
            const uint32_t id = token_of(at, i);
            if constexpr (DTYPE == ANSZP_OUT_BF16) {
                const uint32_t w = id < n ? static_cast<const uint16_t*>(logits)[from + id] : 0xFF80u;
                l.w[i >> 1] = i & 1u ? l.w[i >> 1] | w << 16 : w;
            } else {
                l.w[i >> 2][i & 3u] = id < n ? static_cast<const uint32_t*>(logits)[from + id] : 0xFF800000u;
            }
        }
        return l;
    }
    // work(eight logits, the first one's token) for all tokens.  Several loads are under way together, and none of these looks for the row's end.
    template <class Work>
    __device__ __forceinline__ void each(Work work) const {
        constexpr uint32_t kAtOnce = DTYPE == ANSZP_OUT_BF16 ? 4u : 2u, kLast = 8u / kPiece * kApart - kApart + kPiece;
        uint32_t at = threadIdx.x * kPiece;
        for (; at + (kAtOnce - 1u) * THREADS * 8u + kLast <= n; at += kAtOnce * THREADS * 8u) {
            Eight<DTYPE> l[kAtOnce];
#pragma unroll
            for (uint32_t j = 0; j < kAtOnce; ++j) l[j] = eight(at + j * THREADS * 8u);
#pragma unroll
            for (uint32_t j = 0; j < kAtOnce; ++j) work(l[j], at + j * THREADS * 8u);
        }
        for (; at < n; at += THREADS * 8u) work(at + kLast <= n ? eight(at) : last_eight(at), at);
    }
    __device__ __forceinline__ float logit(uint32_t id) const {
        return DTYPE == ANSZP_OUT_BF16 ? bf16_low(static_cast<const uint16_t*>(logits)[from + id]) : static_cast<const float*>(logits)[from + id];
    }
    // Tokens with logits near `mid` or `mid_b`, by less than `half` and `half_b`, into the list, as many as it holds, by their numbers; sh.listed counts
    // them all.  (What they weigh is worked out behind the pass, by a thread each: here the registers of eight logits would be looked up by number, which is
    // done in memory.  Which lanes have one is known to the whole wavefront: groups that have none, most, are through behind four instructions a logit.)
    __device__ __forceinline__ void list_those(float mid, float half, float mid_b, float half_b) const {
        each([&](const Eight<DTYPE>& l, uint32_t at) __attribute__((always_inline)) {
            uint64_t those[8], any = 0u;
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) {
                those[i] = __ballot(fabsf(l[i] - mid) <= half || fabsf(l[i] - mid_b) <= half_b);
                any |= those[i];
            }
            if (!any) return;
            uint32_t count = 0u, place = 0u;
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) count += uint32_t(__builtin_popcountll(those[i]));
            const uint32_t first = uint32_t(__builtin_ctzll(__ballot(true)));
            if ((threadIdx.x & 63u) == first) place = atomicAdd(&sh.listed, count);
            place = uint32_t(__builtin_amdgcn_readlane(int(place), first));
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) {
                if (!those[i]) continue;
                const uint32_t own = place + __builtin_amdgcn_mbcnt_hi(uint32_t(those[i] >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(those[i]), 0u));
                if (those[i] >> (threadIdx.x & 63u) & 1u && own < kList) sh.list[own].order = token_of(at, i);
                place += uint32_t(__builtin_popcountll(those[i]));
            }
        });
        __syncthreads();
    }
    // This thread's of the n tokens of the list: its order and, where it weighs something, its bin and q.  (What lies behind the row's end was as low as a masked one.)
    __device__ __forceinline__ bool listed_one(uint32_t listed, Entry& e, uint32_t& bin) const {
        if (threadIdx.x >= listed) return false;
        const uint32_t id = uint32_t(sh.list[threadIdx.x].order);
        if (id >= n) return false;
        const float l = logit(id);
        e.order = order_of(key_of(l), id);
        return weigh(l, bin, e.q);
    }
    // work(logit, token) for all tokens, in a short loop: for the passes that few rows need
    template <class Work>
    __device__ __forceinline__ void each_slowly(Work work) const {
        for (uint32_t at = threadIdx.x; at < n; at += THREADS * 4u) {
            float l[4];
#pragma unroll
            for (uint32_t j = 0; j < 4u; ++j) l[j] = logit(uint32_t(least(at + j * THREADS, n - 1u)));
#pragma unroll
            for (uint32_t j = 0; j < 4u; ++j)
                if (at + j * THREADS < n) work(l[j], at + j * THREADS);
        }
    }
    __device__ __forceinline__ void set_scale(float largest, float temperature) {
        constexpr double kLn2 = 0.69314718055994530942 / double(kSteps), kEnd = 0.5 * kLn2;
        top = double(largest);
        steps = 1.4426950408889634074 * double(kSteps) / double(temperature);
        // (a shift that all t of a row share changes nothing but the zero of their scale; where the product is so large that it would, logits are taken from the largest first)
        const double product = top * steps;
        far = !(fabs(product) < 0x1p32);
        shift = far ? 0.0 : product;
        one = __builtin_bit_cast(double, uint64_t(1023u + point) << 52);
        // exp(y ln2 / 64) for |y| <= 1/2 by three powers, to 5e-12: the fourth power's term, x^4 / 24, is spread out as Chebyshev's, x^4 ~ e^2 x^2 - e^4 / 8
        c0 = (1.0 - kEnd * kEnd * kEnd * kEnd / 192.0) * one + 0x1p52;
        c1 = kLn2 * one;
        c2 = kLn2 * kLn2 * (0.5 + kEnd * kEnd / 24.0) * one;
        c3 = kLn2 * kLn2 * kLn2 / 6.0 * one;
    }
    // The bin of a logit and its q; false: it weighs nothing.  (A masked one is infinitely far, or with an infinite temperature no number.)
    __device__ __forceinline__ bool weigh(float l, uint32_t& bin, uint64_t& q) const {
        double v = double(l);
        if (far) v -= top;
        const double t = fma(v, -steps, shift);
        if (!(t < double(kBins) - 0.5)) return false;
        constexpr double kWhole = 0x1.8p52;
        const double whole = t + kWhole, y = (whole - kWhole) - t;
        bin = uint32_t(__builtin_bit_cast(uint64_t, whole));
        q = __builtin_bit_cast(uint64_t, fma(y, fma(y, fma(y, c3, c2), c1), c0)) & 0xFFFFFFFFFFFFFull;
        return true;
    }
    // Logits between which those of bins first .. last surely are, and the same as a middle and how far from it.
    __device__ __forceinline__ void reach_of(uint32_t first, uint32_t last, float& lo, float& hi) const {
        const double by = 1.0 / steps, low = top - (double(last) + 0.5) * by, high = top - (double(first) - 0.5) * by, more = (fabs(top) + fabs(low)) * 0x1p-22 + 1e-30;
        lo = steps > 1e-300 ? float(low - more) : -__builtin_inff();
        hi = steps > 1e-300 ? float(high + more) : __builtin_inff();
    }
    static __device__ __forceinline__ void middle_of(float lo, float hi, float& mid, float& half) {
        const bool finite = lo > -0x1p126f && hi < 0x1p126f;
        mid = finite ? 0.5f * (lo + hi) : 0.0f;
        half = finite ? 0.5f * (hi - lo) + (fabsf(lo) + fabsf(hi)) * 0x1p-22f : __builtin_inff();
    }
    // The sum of `v` over the threads before this one.
    __device__ __forceinline__ uint64_t added_before(uint64_t v, uint64_t* of_wave) const {
        uint64_t upto = v;
        for (uint32_t d = 1; d < 64u; d <<= 1) {
            const uint64_t other = __shfl_up(upto, d);
            if ((threadIdx.x & 63u) >= d) upto += other;
        }
        if ((threadIdx.x & 63u) == 63u) of_wave[threadIdx.x >> 6] = upto;
        __syncthreads();
        uint64_t before = upto - v;
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) {
            const uint64_t other = of_wave[w];
            before += w < threadIdx.x >> 6 ? other : 0u;
        }
        return before;
    }
    __device__ __forceinline__ uint64_t of_all(const uint64_t* of_wave) const {
        uint64_t all = 0u;
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) all += of_wave[w];
        return all;
    }
    // The largest of `v` over all threads.
    __device__ __forceinline__ uint64_t most_of_all(uint64_t v) const {
        for (uint32_t d = 32; d; d >>= 1) {
            const uint64_t other = __shfl_xor(v, d);
            v = other > v ? other : v;
        }
        __syncthreads();
        if ((threadIdx.x & 63u) == 0u) sh.of_wave[threadIdx.x >> 6] = v;
        __syncthreads();
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) v = sh.of_wave[w] > v ? sh.of_wave[w] : v;
        return v;
    }

    // The first token with this logit.  (A pass that counts as it goes, as the next one, takes a sum over the workgroup for every 8192 tokens: 32 us for 131072, this 11.)
    __device__ __forceinline__ uint32_t first_equal(float logit) const {
        uint32_t first = ~0u;
        each([&](const Eight<DTYPE>& l, uint32_t at) __attribute__((always_inline)) {
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) {
                const uint32_t id = l[i] == logit ? token_of(at, i) : ~0u;
                first = id < first ? id : first;
            }
        });
        return ~uint32_t(most_of_all(~first));
    }
    // The token that is the `nth` (from 1 on) of those with this logit.
    __device__ __forceinline__ void find_equal(uint32_t key, uint64_t nth) const {
        uint64_t passed = 0u;
        for (uint32_t first = 0; first < n; first += THREADS * 8u) {
            const uint32_t at = first + threadIdx.x * 8u, there = at < n ? n - at : 0u;
            Eight<DTYPE> l;
            uint32_t mine = 0u;
            if (there) {
                l.load(logits, from + at, there);
                for (uint32_t i = 0; i < 8u; ++i) mine += i < there && key_of(l[i]) == key ? 1u : 0u;
            }
            __syncthreads();
            uint64_t seen = passed + added_before(mine, sh.of_wave);
            passed += of_all(sh.of_wave);
            if (mine)
                for (uint32_t i = 0; i < 8u; ++i)
                    if (i < there && key_of(l[i]) == key && ++seen == nth) sh.found_id = at + i;
            if (passed >= nth) break;
        }
        __syncthreads();
    }

    // What lies before entry `e` among those of its bin in the list (ALIKE: of all): how many, and the sum of what they hold.
    template <bool ALIKE>
    __device__ __forceinline__ void before_in_list(uint32_t listed, const Entry& e, uint32_t bin, uint64_t& count, uint64_t& sum) const {
        uint32_t counted = 0u;
        for (uint32_t j = 0; j < listed; j += 8u) {                  // (the list's entries behind the last are in LDS, too, and not counted)
            Entry other[8];
            uint32_t its[8];
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) {
                other[i] = sh.list[j + i];
                if constexpr (!ALIKE) its[i] = sh.list_bin[j + i];
            }
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) {
                const bool first = other[i].order > e.order && j + i < listed && (ALIKE || its[i] == bin);
                counted += first ? 1u : 0u;
                sum += first ? other[i].q : 0u;
            }
        }
        count += counted;
    }

    // The sums of q (MASSES) and the counts (COUNTS) of all bins made into what lies before each.
    template <bool MASSES, bool COUNTS>
    __device__ __forceinline__ void add_up_bins() const {
        constexpr uint32_t kEach = (kBins + THREADS - 1u) / THREADS;
        uint64_t mass[kEach], masses = 0u, counts = 0u;
        uint32_t count[kEach];
        const uint32_t first = threadIdx.x * kEach;
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
            const bool there = first + i < kBins;
            if constexpr (MASSES) mass[i] = there ? mass_of(height(sh, first + i), sh.mass[first + i]) : 0u;
            if constexpr (COUNTS) count[i] = there ? sh.count[first + i] : 0u;
            if constexpr (MASSES) masses += mass[i];
            if constexpr (COUNTS) counts += count[i];
        }
        uint64_t upto = 0u, counted = 0u;
        if constexpr (MASSES) upto = added_before(masses, sh.of_wave);
        if constexpr (COUNTS) counted = added_before(counts, sh.of_wave_too);
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
            if (first + i <= kBins) {
                if constexpr (MASSES) sh.mass[first + i] = upto;
                if constexpr (COUNTS) sh.count[first + i] = uint32_t(counted);
            }
            if constexpr (MASSES) upto += mass[i];
            if constexpr (COUNTS) counted += count[i];
        }
        __syncthreads();
    }
    // The bin in which some number that rises passes `wanted`: the one with at(bin) < wanted <= at(bin + 1).
    template <class At>
    __device__ __forceinline__ void mark_bin(At at, uint64_t wanted, uint32_t& found) const {
        for (uint32_t b = threadIdx.x; b < kBins; b += THREADS)
            if (at(b) < wanted && wanted <= at(b + 1u)) found = b;
    }
};

// The first token of a bin at which so many tokens are reached (BY_COUNT), or a mass behind what lies before the bin, as the bin as a whole does: its number, its q and the sum
// up to it.
template <bool BY_COUNT, class Row>
__device__ __forceinline__ void find(const Row& row, uint32_t bin, uint64_t wanted) {
    Shared& sh = row.sh;
    const uint64_t mass_before = sh.mass[bin];
    const double high_of = height(sh, bin);
    const auto reach = [=](uint64_t count, uint64_t sum) __attribute__((always_inline)) { return BY_COUNT ? count >= wanted : mass_before + mass_of(high_of, sum) >= wanted; };
    uint32_t least = 0u, most = ~0u;                            // the logits looked at, by their keys
    uint64_t before = 0u, sum_before = 0u;                      // what lies above them in the bin
    float low, high;
    row.reach_of(bin, bin, low, high);
    for (;;) {
        __syncthreads();
        if (threadIdx.x == 0u) {
            sh.listed = 0u;
            sh.least = ~0u;
            sh.most = 0u;
        }
        __syncthreads();
        row.each_slowly([&](float l, uint32_t id) __attribute__((always_inline)) {
            if (!(l >= low && l <= high)) return;
            uint32_t b;
            uint64_t q;
            if (!row.weigh(l, b, q) || b != bin) return;
            const uint32_t key = key_of(l);
            if (key < least || key > most) return;
            const uint32_t at = atomicAdd(&sh.listed, 1u);
            if (at < kList) sh.list[at] = {order_of(key, id), q};
            atomicMin(&sh.least, key);
            atomicMax(&sh.most, key);
        });
        __syncthreads();
        const uint32_t there = sh.listed;
        least = sh.least;
        most = sh.most;
        if (there <= kList) {
            if (threadIdx.x < there) {
                const Entry e = sh.list[threadIdx.x];
                uint64_t count = before, sum = sum_before;
                row.template before_in_list<true>(there, e, bin, count, sum);
                if (!reach(count, sum) && reach(count + 1u, sum + e.q)) {
                    sh.found_id = id_of(e);
                    sh.found_q = e.q;
                    sh.found_sum = sum + e.q;
                }
            }
            __syncthreads();
            return;
        }
        if (least == most) {
            // Equal logits: which of them it is, then where that one is.
            const uint64_t q = sh.list[0].q;
            uint32_t under = 0u, over = there;                  // reach holds for `over` of them, not for `under`
            while (over - under > 1u) {
                const uint32_t mid = under + (over - under) / 2u;
                if (reach(before + mid, sum_before + mid * q)) over = mid;
                else under = mid;
            }
            row.find_equal(most, over);
            if (threadIdx.x == 0u) {
                sh.found_q = q;
                sh.found_sum = sum_before + over * q;
            }
            __syncthreads();
            return;
        }
        // Too many: cut between the least and the largest key.
        static_assert(kCuts <= Row::kWaves * 64u, "a cut a thread");
        const uint64_t range = uint64_t(most) - least + 1u;
        if (threadIdx.x < kCuts) {
            sh.cut_sum[threadIdx.x] = 0u;
            sh.cut_count[threadIdx.x] = 0u;
        }
        __syncthreads();
        row.each_slowly([&](float l, uint32_t) __attribute__((always_inline)) {
            if (!(l >= low && l <= high)) return;
            uint32_t b;
            uint64_t q;
            if (!row.weigh(l, b, q) || b != bin) return;
            const uint32_t key = key_of(l);
            if (key < least || key > most) return;
            const uint32_t cut = uint32_t(uint64_t(most - key) * kCuts / range);
            atomicAdd(reinterpret_cast<unsigned long long*>(&sh.cut_sum[cut]), q);
            atomicAdd(&sh.cut_count[cut], 1u);
        });
        __syncthreads();
        const bool cuts = threadIdx.x < kCuts;
        const uint64_t count = cuts ? sh.cut_count[threadIdx.x] : 0u, sum = cuts ? sh.cut_sum[threadIdx.x] : 0u;
        const uint64_t count_upto = before + row.added_before(count, sh.of_wave), sum_upto = sum_before + row.added_before(sum, sh.of_wave_too);
        if (cuts && !reach(count_upto, sum_upto) && reach(count_upto + count, sum_upto + sum)) {
            sh.found = threadIdx.x;
            sh.found_count = count_upto;
            sh.found_sum = sum_upto;
        }
        __syncthreads();
        // the keys whose cut is `found`
        const uint64_t cut = sh.found, nearest = (cut * range + kCuts - 1u) / kCuts, furthest = ((cut + 1u) * range + kCuts - 1u) / kCuts - 1u;
        before = sh.found_count;
        sum_before = sh.found_sum;
        least = uint32_t(most - furthest);
        most = uint32_t(most - nearest);
    }
}

struct Settings {
    float u, top_p, min_p;
    uint32_t top_k;                     // 0: all
};
// What part of the kept mass is passed, and the least mass that reaches top_p of all.
__device__ __forceinline__ uint64_t drawn_at(float u, uint64_t kept) {
    const uint64_t at = u > 0.0f ? u < 1.0f ? uint64_t(double(u) * double(kept)) : kept - 1u : 0u;
    return at < kept ? at : kept - 1u;
}
__device__ __forceinline__ uint64_t wanted_of(float top_p, uint64_t all) {
    const uint64_t wanted = top_p > 0.0f ? uint64_t(ceil(double(top_p) * double(all))) : 1u;
    return wanted < 1u ? 1u : wanted > all ? all : wanted;
}

template <uint32_t DTYPE, uint32_t THREADS>
__global__ __launch_bounds__(THREADS, 4) void sample_kernel(SampleParams p) {
    __shared__ Shared sh;
    const uint64_t r = uint64_t(blockIdx.y) * kAcross + blockIdx.x;
    if (r >= p.rows) return;
    const float temperature = p.temperature ? p.temperature[r] : p.any_temperature;
    const int32_t top_k = p.top_k ? p.top_k[r] : p.any_top_k;
    const Settings set = {p.uniforms[r], p.top_p ? p.top_p[r] : p.any_top_p, p.min_p ? p.min_p[r] : p.any_min_p, top_k > 0 ? uint32_t(top_k) : 0u};
    Row<DTYPE, THREADS> row = {sh, p.logits, r * p.stride, p.vocabulary, p.point};
    const auto answer = [&](int64_t token, float chance) __attribute__((always_inline)) {
        if (threadIdx.x != 0u) return;
        p.tokens[r] = token;
        if (p.chances) p.chances[r] = chance;
    };
    const auto clear = [&]() __attribute__((always_inline)) {
        for (uint32_t i = threadIdx.x; i <= kBins; i += THREADS) {
            sh.mass[i] = 0u;
            sh.count[i] = 0u;
        }
        if (threadIdx.x == 0u) sh.listed = 0u;
    };
    clear();
    if (threadIdx.x < kSteps) sh.octave[threadIdx.x] = exp2(double(threadIdx.x) * (-1.0 / double(kSteps)));

    // The largest logit; the largest of bits without sign is a NaN's where there is one.
    float top = -__builtin_inff();
    uint32_t bits = 0u;
    row.each([&](const Eight<DTYPE>& l, uint32_t) __attribute__((always_inline)) {
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) {
            top = fmaxf(top, l[i]);
            const uint32_t w = __builtin_bit_cast(uint32_t, l[i]) & 0x7FFFFFFFu;
            bits = w > bits ? w : bits;
        }
    });
    const float own_top = top;
    {
        const uint64_t both = uint64_t(most_of_wave(key_of(top))) << 32 | most_of_wave(bits);
        if ((threadIdx.x & 63u) == 0u) sh.of_wave[threadIdx.x >> 6] = both;
    }
    __syncthreads();
    uint32_t best = 0u;
#pragma unroll
    for (uint32_t w = 0; w < THREADS / 64u; ++w) {
        const uint64_t both = sh.of_wave[w];
        best = uint32_t(both >> 32) > best ? uint32_t(both >> 32) : best;
        bits = uint32_t(both) > bits ? uint32_t(both) : bits;
    }
    top = of_key(best);
    if (bits > 0x7F800000u || !(temperature >= 0.0f) || top == -__builtin_inff()) {
        answer(-1, 0.0f);
        return;
    }
    if (temperature == 0.0f || set.top_k == 1u) {
        answer(int64_t(row.first_equal(top)), 1.0f);
        return;
    }
    if (top == __builtin_inff()) {
        // infinities share the row alone, each a mass of 1
        uint32_t mine = 0u;
        row.each([&](const Eight<DTYPE>& l, uint32_t) __attribute__((always_inline)) {
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) mine += l[i] == __builtin_inff() ? 1u : 0u;
        });
        __syncthreads();
        row.added_before(mine, sh.of_wave);
        uint64_t kept = row.of_all(sh.of_wave);
        kept = set.top_k && set.top_k < kept ? set.top_k : kept;
        if (set.top_p < 1.0f) kept = wanted_of(set.top_p, kept);
        row.find_equal(best, drawn_at(set.u, kept) + 1u);
        answer(int64_t(sh.found_id), float(1.0 / double(kept)));
        return;
    }
    row.set_scale(top, temperature);
    // min_p of what the largest weighs (not looked at where there is no min_p)
    const double least = set.min_p < 1.0f ? double(set.min_p) : 1.0;
    uint32_t its_bin = 0u;
    uint64_t its_q = 0u;
    row.weigh(top, its_bin, its_q);
    const double border = least * double(its_q);

    // Few tokens that may be kept are listed, and all else is done in the list.  top_k: as many threads' largest logits are at least the least of those that are
    // listed, so that at least top_k tokens are.  min_p alone: those that weigh enough.
    const bool few = set.top_k && set.top_k <= kList / 2u, by_weight = set.min_p > 0.0f && !(set.top_p < 1.0f);
    if (few || by_weight) {
        uint32_t last = kBins - 1u;
        if (few) {
            uint32_t bin;
            uint64_t q;
            if (row.weigh(own_top, bin, q)) atomicAdd(&sh.count[bin], 1u);
            __syncthreads();
            row.template add_up_bins<false, true>();
            if (set.top_k <= sh.count[kBins]) {
                row.mark_bin([&](uint32_t i) __attribute__((always_inline)) { return uint64_t(sh.count[i]); }, set.top_k, sh.found);
                __syncthreads();
                last = sh.found;
            }
        }
        if (by_weight) {
            const double t = -double(kSteps) * log2(least) + 1.0;
            last = t < double(last) ? uint32_t(t) : last;
        }
        float low, high;
        row.reach_of(0u, last, low, high);
        float mid, half;
        row.middle_of(low, top, mid, half);
        row.list_those(mid, half, mid, half);
        const uint32_t n = sh.listed;
        if (n <= kList) {
            uint64_t count = 0u, before = 0u;
            Entry e = {0u, 0u};
            uint32_t bin = 0u;
            const bool there = row.listed_one(n, e, bin);
            // (its weight as the way over the bins has it: of a light token the mass, a whole number, has few digits)
            const double weight = there ? height(sh, bin) * double(e.q) : 0.0;
            e.q = uint64_t(weight);
            __syncthreads();
            if (threadIdx.x < n) sh.list[threadIdx.x] = e;
            const uint32_t those = uint32_t(__syncthreads_count(there));
            if (there) row.template before_in_list<true>(n, e, 0u, count, before);
            if (there && count == (set.top_k && set.top_k < those ? set.top_k : those) - 1u) sh.found_sum = before + e.q;
            __syncthreads();
            const uint64_t all = sh.found_sum;
            uint64_t kept = all;
            if (set.top_p < 1.0f) {
                const uint64_t wanted = wanted_of(set.top_p, all);
                if (there && before < wanted && wanted <= before + e.q) sh.found_count = before + e.q;
                __syncthreads();
                kept = sh.found_count;
            }
            if (set.min_p > 0.0f) {
                // (those that weigh enough are the first of the order: the last one's sum is theirs)
                const uint64_t upto = row.most_of_all(there && weight >= border ? before + e.q : 0u);
                kept = upto < kept ? upto : kept;
            }
            const uint64_t at = drawn_at(set.u, kept);
            if (there && before <= at && at < before + e.q) {
                p.tokens[r] = int64_t(id_of(e));
                if (p.chances) p.chances[r] = float(weight / double(kept));
            }
            return;
        }
        __syncthreads();
        clear();
        __syncthreads();
    }

    const bool counts = set.top_k != 0u;
    row.each([&](const Eight<DTYPE>& l, uint32_t) __attribute__((always_inline)) {
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) {
            uint32_t bin;
            uint64_t q;
            if (row.weigh(l[i], bin, q)) {
                atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[bin]), q);
                if (counts) atomicAdd(&sh.count[bin], 1u);
            }
            __builtin_amdgcn_sched_barrier(0);                      // (side by side they take registers that the wavefronts have not)
        }
    });
    __syncthreads();
    if (counts) row.template add_up_bins<true, true>();
    else row.template add_up_bins<true, false>();
    const auto mass_before = [&](uint32_t b) __attribute__((always_inline)) { return sh.mass[b]; };

    uint64_t kept = sh.mass[kBins];
    if (set.top_k && set.top_k < sh.count[kBins]) {
        row.mark_bin([&](uint32_t i) __attribute__((always_inline)) { return uint64_t(sh.count[i]); }, set.top_k, sh.found);
        __syncthreads();
        const uint32_t b = sh.found;
        const uint64_t wanted = set.top_k - sh.count[b];
        if (wanted == sh.count[b + 1u] - sh.count[b]) {
            kept = sh.mass[b + 1u];
        } else {
            find<true>(row, b, wanted);
            kept = sh.mass[b] + mass_of(height(sh, b), sh.found_sum);
        }
        __syncthreads();
    }
    // The bins in which the two other borders are, and the least and the most that they leave: the first border counts, and where both are in a bin both
    // have to be worked out.
    uint32_t bin_p = kBins, bin_m = kBins;
    uint64_t wanted = 0u, fewest = kept, most = kept;
    if (set.top_p < 1.0f) {
        wanted = wanted_of(set.top_p, kept);
        row.mark_bin(mass_before, wanted, sh.found_top_p);
        __syncthreads();
        bin_p = sh.found_top_p;
    }
    if (set.min_p > 0.0f) {
        const double t = -double(kSteps) * log2(least);
        if (t < double(kBins) - 1.0) bin_m = uint32_t(rint(t));
    }
    if (bin_p > bin_m) bin_p = kBins;
    if (bin_m > bin_p) bin_m = kBins;
    const uint32_t bin_b = bin_p < bin_m ? bin_p : bin_m;
    if (bin_b < kBins) {
        // (top_p's border leaves at least a token of its bin, the weight's perhaps none: then what lies before the bin is all that is kept)
        const uint64_t before = sh.mass[bin_b], some = bin_m == kBins || before == 0u ? before + 1u : before;
        fewest = some < kept ? some : kept;
        most = sh.mass[bin_b + 1u] < kept ? sh.mass[bin_b + 1u] : kept;
    }
    // What is drawn lies in bins first .. last.  Their tokens and those of the border's bin are listed in one go, if they are few.
    row.mark_bin(mass_before, drawn_at(set.u, fewest) + 1u, sh.found);
    row.mark_bin(mass_before, drawn_at(set.u, most) + 1u, sh.found_too);
    if (threadIdx.x == 0u) sh.listed = 0u;
    __syncthreads();
    const uint32_t first = sh.found, last = sh.found_too;
    float low, high, low_b = __builtin_inff(), high_b = -__builtin_inff();
    row.reach_of(first, last, low, high);
    if (bin_b < kBins) row.reach_of(bin_b, bin_b, low_b, high_b);
    float mid, half, mid_b = 0.0f, half_b = -1.0f;
    row.middle_of(low, high, mid, half);
    if (bin_b < kBins) row.middle_of(low_b, high_b, mid_b, half_b);
    row.list_those(mid, half, mid_b, half_b);
    const uint32_t n = sh.listed;
    if (n <= kList) {
        Entry e = {0u, 0u};
        uint32_t bin = 0u;
        uint64_t before = 0u, upto = 0u;
        // (a neighbouring bin's token, of which the list has not all, is none's)
        const bool listed = row.listed_one(n, e, bin) && ((bin >= first && bin <= last) || bin == bin_b);
        __syncthreads();
        if (threadIdx.x < n) {
            sh.list[threadIdx.x] = e;
            sh.list_bin[threadIdx.x] = listed ? bin : ~0u;
        }
        __syncthreads();
        if (listed) {
            uint64_t count = 0u, sum = 0u;
            row.template before_in_list<false>(n, e, bin, count, sum);
            const double high_of = height(sh, bin);
            before = sh.mass[bin] + mass_of(high_of, sum);
            upto = sh.mass[bin] + mass_of(high_of, sum + e.q);
        }
        if (bin_p < kBins) {
            if (listed && bin == bin_p && before < wanted && wanted <= upto) sh.found_sum = upto;
            __syncthreads();
            kept = sh.found_sum < kept ? sh.found_sum : kept;
        }
        if (bin_m < kBins) {
            uint64_t some = row.most_of_all(listed && bin == bin_m && height(sh, bin) * double(e.q) >= border ? upto : 0u);
            some = some > sh.mass[bin_m] ? some : sh.mass[bin_m];
            kept = some < kept ? some : kept;
        }
        const uint64_t at = drawn_at(set.u, kept);
        if (listed && before <= at && at < upto) {
            p.tokens[r] = int64_t(id_of(e));
            if (p.chances) p.chances[r] = float(height(sh, bin) * double(e.q) / double(kept));
        }
        return;
    }
    if (bin_p < kBins) {
        find<false>(row, bin_p, wanted);
        const uint64_t upto = sh.mass[bin_p] + mass_of(height(sh, bin_p), sh.found_sum);
        kept = upto < kept ? upto : kept;
        __syncthreads();
    }
    if (bin_m < kBins) {
        const double high_of = height(sh, bin_m);
        uint64_t sum = 0u;
        row.each_slowly([&](float l, uint32_t) __attribute__((always_inline)) {
            if (!(l >= low_b && l <= high_b)) return;
            uint32_t bin;
            uint64_t q;
            if (row.weigh(l, bin, q) && bin == bin_m && high_of * double(q) >= border) sum += q;
        });
        __syncthreads();
        row.added_before(sum, sh.of_wave);
        const uint64_t upto = sh.mass[bin_m] + mass_of(high_of, row.of_all(sh.of_wave));
        kept = upto < kept ? upto : kept;
        __syncthreads();
    }
    const uint64_t at = drawn_at(set.u, kept);
    row.mark_bin(mass_before, at + 1u, sh.found);
    __syncthreads();
    const uint32_t b = sh.found;
    find<false>(row, b, at + 1u);
    answer(int64_t(sh.found_id), float(height(sh, b) * double(sh.found_q) / double(kept)));
}

template <uint32_t DTYPE>
void launch(const SampleParams& p, hipStream_t s) {
    const dim3 grid(groups_across(p.rows), groups_down(p.rows));
    // More rows than compute units: half the threads, so that a CU has two rows at a time and goes on with one where the other waits.  (512 rows of 131072
    // in bf16 88 us, with 1024 threads 103; 32 rows of 131072 52 us with 1024 threads, 68 with 512; short rows take the same.)
    if (p.rows > device_cus()) hipLaunchKernelGGL((sample_kernel<DTYPE, 512u>), grid, dim3(512), 0, s, p);
    else hipLaunchKernelGGL((sample_kernel<DTYPE, 1024u>), grid, dim3(1024), 0, s, p);
}

}  // namespace

extern "C" int anszp_sample(const anszp_sample_args_t* a, void* hip_stream) {
    if (!a) return ANSZP_E_NULL;
    const auto setting = [](const float* each, float all) { return each || all >= 0.0f; };              // (no NaN either)
    if ((a->dtype != ANSZP_OUT_F32 && a->dtype != ANSZP_OUT_BF16) || a->vocabulary == 0 || a->vocabulary > 1u << 24 || a->rows >= 1ull << 31 ||
        !setting(a->temperatures, a->temperature) || !setting(a->top_ps, a->top_p) || !setting(a->min_ps, a->min_p) || (!a->top_ks && a->top_k < 0))
        return ANSZP_E_RANGE;
    if (a->rows == 0) return ANSZP_OK;
    if (!a->logits || !a->uniforms || !a->tokens) return ANSZP_E_NULL;
    const uint64_t size = a->dtype == ANSZP_OUT_BF16 ? 2u : 4u;
    const Rows logits = {a->logits, a->rows, a->logits_stride * size, a->vocabulary * size}, tokens = {a->tokens, 1, 0, a->rows * 8u}, chances = {a->chances, 1, 0, a->rows * 4u};
    if (meet(tokens, logits) || meet(chances, logits) || meet(tokens, chances)) return ANSZP_E_RANGE;
    for (const void* each : {static_cast<const void*>(a->uniforms), static_cast<const void*>(a->temperatures), static_cast<const void*>(a->top_ks),
                             static_cast<const void*>(a->top_ps), static_cast<const void*>(a->min_ps)})
        if (meet(tokens, {each, 1, 0, a->rows * 4u}) || meet(chances, {each, 1, 0, a->rows * 4u})) return ANSZP_E_RANGE;
    uint32_t digits = 0u;                                           // sums of q over all tokens are below 2^63
    while (1ull << digits < a->vocabulary) ++digits;
    SampleParams p = {a->logits, a->uniforms, a->temperatures, a->top_ks, a->top_ps, a->min_ps, a->tokens, a->chances, a->rows, a->logits_stride, a->vocabulary, a->top_k,
                      a->temperature, a->top_p, a->min_p, digits > 18u ? 62u - digits : 44u};
    if (a->dtype == ANSZP_OUT_F32) launch<ANSZP_OUT_F32>(p, static_cast<hipStream_t>(hip_stream));
    else launch<ANSZP_OUT_BF16>(p, static_cast<hipStream_t>(hip_stream));
    return hipGetLastError() == hipSuccess ? ANSZP_OK : ANSZP_E_HIP;
}
