// The next token of each row drawn from its logits, for gfx950.  With l the logits, tokens in the order of falling l (equal ones: the lower first) and
//   w = exp((l - max l) / temperature)
// a row keeps the shortest of these beginnings of the order: the first top_k; of those the shortest whose weights reach top_p of theirs; the ones with
// w >= min_p.  It draws the first token at which the sum of the kept weights passes uniform * (their sum).
//
// Sums decide which token it is, so they are whole numbers and no order of additions changes them.  With t = 64 log2(e) (max l - l) / temperature, in 64
// bits, and b = round(t):
//   w = 2^(-b / 64) * q,    q = 2^((b - t) / 64) in 1 +- 0.0054, which four terms of its series give to 4e-14,
// the q are held in fixed point with 2^-44 (less only for more than 2^18 tokens) and added up for each b in LDS; a bin's mass is its sum times 2^(-b / 64), rounded down, and
// masses are added up over the bins.  What is further down than 44 octaves weighs nothing.  A border that lies in a bin is found among the bin's own
// tokens, every one compared with all others; where a bin has more than the list holds, it is cut by its tokens' own logits first, as often as that takes.
#include <hip/hip_runtime.h>

#include "anszp_numbers.h"

namespace {

constexpr uint32_t kThreads = 1024, kWaves = kThreads / 64u, kSteps = 64, kBins = 44u * kSteps, kList = 1024, kCuts = 1024;

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

struct Shared {
    uint64_t mass[kBins + 1u];          // first the sums of q, then the masses before each bin
    uint32_t count[kBins + 1u];         // first the tokens, then those before each bin
    uint64_t cut_sum[kCuts];
    uint32_t cut_count[kCuts];
    uint32_t list_key[kList], list_id[kList];
    uint64_t list_q[kList];             // q, or a mass
    uint64_t of_wave[kWaves], of_wave_too[kWaves];
    uint32_t listed, least, most, list_bin;
    uint32_t found, found_id;
    uint64_t found_sum, found_q, found_count;
};

template <uint32_t DTYPE>
struct Row {
    const void* logits;
    uint64_t from;
    uint32_t n, point;
    double top, steps;                  // the largest logit, 64 log2(e) / temperature

    // work(logit, token) for all tokens; a thread's come in rising order
    template <class Work>
    __device__ __forceinline__ void each(Work work) const {
        uint32_t at = threadIdx.x * 8u;
        for (; at + kThreads * 8u + 8u <= n; at += kThreads * 16u) {                // (two loads under way)
            Eight<DTYPE> l, m;
            l.load(logits, from + at, 8u);
            m.load(logits, from + at + kThreads * 8u, 8u);
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) work(l[i], at + i);
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) work(m[i], at + kThreads * 8u + i);
        }
        for (; at < n; at += kThreads * 8u) {
            const uint32_t there = n - at;
            Eight<DTYPE> l;
            l.load(logits, from + at, there);
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i)
                if (i < there) work(l[i], at + i);
        }
    }
    // The bin of a logit and its q; false: it weighs nothing.  (A masked one is infinitely far, or with an infinite temperature no number.)
    __device__ __forceinline__ bool weigh(float l, uint32_t& bin, uint64_t& q) const {
        const double t = (top - double(l)) * steps;
        if (!(t < double(kBins) - 0.5)) return false;
        constexpr double kWhole = 0x1.8p52, kLn2 = 0.69314718055994530942 / double(kSteps);
        const double whole = t + kWhole, y = (whole - kWhole) - t, one = __builtin_bit_cast(double, uint64_t(1023u + point) << 52);
        bin = uint32_t(__builtin_bit_cast(uint64_t, whole));
        // exp(y ln2 / 64) without its 1, times 2^point
        double s = fma(y, kLn2 * kLn2 * kLn2 * kLn2 / 24.0, kLn2 * kLn2 * kLn2 / 6.0);
        s = fma(y, s, kLn2 * kLn2 / 2.0);
        s = fma(y, s, kLn2);
        q = __builtin_bit_cast(uint64_t, fma(s, y * one, one + 0x1p52)) & 0xFFFFFFFFFFFFFull;
        return true;
    }
    // Logits between which those of bins first .. last surely are.
    __device__ __forceinline__ void reach_of(uint32_t first, uint32_t last, float& lo, float& hi) const {
        const double low = top - (double(last) + 0.5) / steps, high = top - (double(first) - 0.5) / steps, more = (fabs(top) + fabs(low)) * 0x1p-22 + 1e-30;
        lo = steps > 1e-300 ? float(low - more) : -__builtin_inff();
        hi = steps > 1e-300 ? float(high + more) : __builtin_inff();
    }
};

__device__ __forceinline__ double height(uint32_t bin) { return exp2(double(bin) * (-1.0 / double(kSteps))); }
__device__ __forceinline__ uint64_t mass_of(double height, uint64_t sum) { return uint64_t(height * double(sum)); }

// The sum of `v` over the threads before this one.
__device__ __forceinline__ uint64_t added_before(uint64_t v, uint64_t* of_wave) {
    uint64_t upto = v;
    for (uint32_t d = 1; d < 64u; d <<= 1) {
        const uint64_t other = __shfl_up(upto, d);
        if ((threadIdx.x & 63u) >= d) upto += other;
    }
    if ((threadIdx.x & 63u) == 63u) of_wave[threadIdx.x >> 6] = upto;
    __syncthreads();
    uint64_t before = upto - v;
    for (uint32_t w = 0; w < kWaves; ++w)
        if (w < threadIdx.x >> 6) before += of_wave[w];
    return before;
}

// The token that is the `nth` (from 1 on) of those with this logit.
template <uint32_t DTYPE>
__device__ void find_equal(Shared& sh, const Row<DTYPE>& row, uint32_t key, uint64_t nth) {
    uint64_t passed = 0u;
    for (uint32_t from = 0; from < row.n; from += kThreads * 8u) {
        const uint32_t at = from + threadIdx.x * 8u, there = at < row.n ? row.n - at : 0u;
        Eight<DTYPE> l;
        uint32_t mine = 0u;
        if (there) {
            l.load(row.logits, row.from + at, there);
            for (uint32_t i = 0; i < 8u; ++i) mine += i < there && key_of(l[i]) == key ? 1u : 0u;
        }
        __syncthreads();
        uint64_t seen = passed + added_before(mine, sh.of_wave);
        for (uint32_t w = 0; w < kWaves; ++w) passed += sh.of_wave[w];
        if (mine)
            for (uint32_t i = 0; i < 8u; ++i)
                if (i < there && key_of(l[i]) == key && ++seen == nth) sh.found_id = at + i;
    }
    __syncthreads();
}

// What lies before the list's entry `own` in the order of logits: how many of the n entries, and the sum of what they hold.
__device__ __forceinline__ void before_in_list(const Shared& sh, uint32_t n, uint32_t own, uint64_t& count, uint64_t& sum) {
    const uint32_t key = sh.list_key[own], id = sh.list_id[own];
    uint32_t counted = 0u;
    for (uint32_t j = 0; j < n; ++j) {
        const uint32_t other = sh.list_key[j];
        const bool first = other > key || (other == key && sh.list_id[j] < id);
        counted += first ? 1u : 0u;
        sum += first ? sh.list_q[j] : 0u;
    }
    count += counted;
}

// The first token of a bin at which reach(tokens up to it, their sum of q) holds, which it does for the bin as a whole: its number, its q and the sum.
template <uint32_t DTYPE, class Reach>
__device__ __forceinline__ void find(Shared& sh, const Row<DTYPE>& row, uint32_t bin, Reach reach) {
    uint32_t lo = 0u, hi = ~0u;                                     // the logits looked at, by their keys
    uint64_t before = 0u, sum_before = 0u;                          // what lies above them in the bin
    float low, high;
    row.reach_of(bin, bin, low, high);
    for (;;) {
        __syncthreads();
        if (sh.list_bin != bin || sh.listed > kList) {
            __syncthreads();
            if (threadIdx.x == 0u) {
                sh.listed = 0u;
                sh.least = ~0u;
                sh.most = 0u;
                sh.list_bin = bin;
            }
            __syncthreads();
            row.each([&](float l, uint32_t id) __attribute__((always_inline)) {
                if (!(l >= low && l <= high)) return;
                uint32_t b;
                uint64_t q;
                if (!row.weigh(l, b, q) || b != bin) return;
                const uint32_t key = key_of(l);
                if (key < lo || key > hi) return;
                const uint32_t at = atomicAdd(&sh.listed, 1u);
                if (at < kList) {
                    sh.list_key[at] = key;
                    sh.list_id[at] = id;
                    sh.list_q[at] = q;
                }
                atomicMin(&sh.least, key);
                atomicMax(&sh.most, key);
            });
            __syncthreads();
        }
        const uint32_t n = sh.listed, least = sh.least, most = sh.most;
        if (n <= kList) {
            if (threadIdx.x < n) {
                uint64_t count = before, sum = sum_before;
                before_in_list(sh, n, threadIdx.x, count, sum);
                const uint64_t q = sh.list_q[threadIdx.x];
                if (!reach(count, sum) && reach(count + 1u, sum + q)) {
                    sh.found_id = sh.list_id[threadIdx.x];
                    sh.found_q = q;
                    sh.found_sum = sum + q;
                }
            }
            if (threadIdx.x == 0u && (lo || ~hi)) sh.list_bin = ~0u;    // (a part of a bin is no bin's list)
            __syncthreads();
            return;
        }
        if (least == most) {
            // Equal logits: which of them it is, then where that one is.
            const uint64_t q = sh.list_q[0];
            uint32_t under = 0u, over = n;                          // reach holds for `over` of them, not for `under`
            while (over - under > 1u) {
                const uint32_t mid = under + (over - under) / 2u;
                if (reach(before + mid, sum_before + mid * q)) over = mid;
                else under = mid;
            }
            find_equal(sh, row, most, over);
            if (threadIdx.x == 0u) {
                sh.found_q = q;
                sh.found_sum = sum_before + over * q;
                sh.list_bin = ~0u;
            }
            __syncthreads();
            return;
        }
        // Too many: cut between the least and the largest key.
        const uint64_t range = uint64_t(most) - least + 1u;
        for (uint32_t i = threadIdx.x; i < kCuts; i += kThreads) {
            sh.cut_sum[i] = 0u;
            sh.cut_count[i] = 0u;
        }
        __syncthreads();
        row.each([&](float l, uint32_t) __attribute__((always_inline)) {
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
        static_assert(kCuts == kThreads, "a cut a thread");
        const uint64_t count = sh.cut_count[threadIdx.x], sum = sh.cut_sum[threadIdx.x];
        const uint64_t count_upto = before + added_before(count, sh.of_wave), sum_upto = sum_before + added_before(sum, sh.of_wave_too);
        if (!reach(count_upto, sum_upto) && reach(count_upto + count, sum_upto + sum)) {
            sh.found = threadIdx.x;
            sh.found_count = count_upto;
            sh.found_sum = sum_upto;
        }
        __syncthreads();
        // the keys whose cut is `found`
        const uint64_t cut = sh.found, nearest = (cut * range + kCuts - 1u) / kCuts, furthest = ((cut + 1u) * range + kCuts - 1u) / kCuts - 1u;
        before = sh.found_count;
        sum_before = sh.found_sum;
        hi = uint32_t(most - nearest);
        lo = uint32_t(most - furthest);
        if (threadIdx.x == 0u) sh.list_bin = ~0u;
    }
}

// The sums of q (or none) and counts of all bins made into what lies before each.
__device__ __forceinline__ void add_up_bins(Shared& sh) {
    constexpr uint32_t kEach = (kBins + kThreads - 1u) / kThreads;
    uint64_t mass[kEach], masses = 0u, counts = 0u;
    uint32_t count[kEach];
    const uint32_t first = threadIdx.x * kEach;
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const bool there = first + i < kBins;
        mass[i] = there ? mass_of(height(first + i), sh.mass[first + i]) : 0u;
        count[i] = there ? sh.count[first + i] : 0u;
        masses += mass[i];
        counts += count[i];
    }
    __syncthreads();
    uint64_t upto = added_before(masses, sh.of_wave), counted = added_before(counts, sh.of_wave_too);
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        if (first + i <= kBins) {
            sh.mass[first + i] = upto;
            sh.count[first + i] = uint32_t(counted);
        }
        upto += mass[i];
        counted += count[i];
    }
    __syncthreads();
}
// The bin in which some number that rises passes `wanted`: the one with at(bin) < wanted <= at(bin + 1).
template <class At>
__device__ __forceinline__ uint32_t bin_of(Shared& sh, At at, uint64_t wanted) {
    for (uint32_t b = threadIdx.x; b < kBins; b += kThreads)
        if (at(b) < wanted && wanted <= at(b + 1u)) sh.found = b;
    __syncthreads();
    const uint32_t b = sh.found;
    __syncthreads();
    return b;
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

// From the list of all tokens that may be kept (key, id, mass), n of them.
__device__ __forceinline__ void draw_from_list(Shared& sh, const Settings& set, uint32_t n, uint32_t point, double least_mass) {
    uint64_t count = 0u, before = 0u, mass = 0u;
    const bool there = threadIdx.x < n;
    if (there) {
        before_in_list(sh, n, threadIdx.x, count, before);
        mass = sh.list_q[threadIdx.x];
    }
    const uint32_t last = (set.top_k && set.top_k < n ? set.top_k : n) - 1u;
    if (there && count == last) sh.found_sum = before + mass;
    __syncthreads();
    const uint64_t all = sh.found_sum;
    uint64_t kept = all;
    if (set.top_p < 1.0f) {
        const uint64_t wanted = wanted_of(set.top_p, all);
        if (there && before < wanted && wanted <= before + mass) sh.found_count = before + mass;
        __syncthreads();
        kept = sh.found_count;
    }
    if (set.min_p > 0.0f) {
        // (those that weigh enough are the first of the order: the last one's sum is theirs)
        uint64_t upto = there && double(mass) >= least_mass ? before + mass : 0u;
        for (uint32_t d = 32; d; d >>= 1) {
            const uint64_t other = __shfl_xor(upto, d);
            upto = other > upto ? other : upto;
        }
        if ((threadIdx.x & 63u) == 0u) sh.of_wave[threadIdx.x >> 6] = upto;
        __syncthreads();
        upto = 0u;
        for (uint32_t w = 0; w < kWaves; ++w) upto = sh.of_wave[w] > upto ? sh.of_wave[w] : upto;
        kept = upto < kept ? upto : kept;
    }
    const uint64_t at = drawn_at(set.u, kept);
    if (there && before <= at && at < before + mass) {
        sh.found_id = sh.list_id[threadIdx.x];
        sh.found_q = mass;
        sh.found_sum = kept;
    }
    __syncthreads();
}

template <uint32_t DTYPE>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleParams p) {
    __shared__ Shared sh;
    const uint64_t r = uint64_t(blockIdx.y) * kAcross + blockIdx.x;
    if (r >= p.rows) return;
    const float temperature = p.temperature ? p.temperature[r] : p.any_temperature;
    const int32_t top_k = p.top_k ? p.top_k[r] : p.any_top_k;
    const Settings set = {p.uniforms[r], p.top_p ? p.top_p[r] : p.any_top_p, p.min_p ? p.min_p[r] : p.any_min_p, top_k > 0 ? uint32_t(top_k) : 0u};
    Row<DTYPE> row = {p.logits, r * p.stride, p.vocabulary, p.point, 0.0, 0.0};
    const auto answer = [&](int64_t token, float chance) __attribute__((always_inline)) {
        if (threadIdx.x != 0u) return;
        p.tokens[r] = token;
        if (p.chances) p.chances[r] = chance;
    };

    // The largest logit; the largest of bits without sign is a NaN's where there is one.
    float top = -__builtin_inff();
    uint32_t bits = 0u;
    row.each([&](float l, uint32_t) __attribute__((always_inline)) {
        top = fmaxf(top, l);
        const uint32_t w = __builtin_bit_cast(uint32_t, l) & 0x7FFFFFFFu;
        bits = w > bits ? w : bits;
    });
    const float own_top = top;
    uint64_t both = uint64_t(key_of(top)) << 32 | bits;
    for (uint32_t d = 32; d; d >>= 1) {
        const uint64_t other = __shfl_xor(both, d);
        both = (other >> 32 > both >> 32 ? other >> 32 : both >> 32) << 32 | (uint32_t(other) > uint32_t(both) ? uint32_t(other) : uint32_t(both));
    }
    if ((threadIdx.x & 63u) == 0u) sh.of_wave[threadIdx.x >> 6] = both;
    for (uint32_t i = threadIdx.x; i <= kBins; i += kThreads) {
        sh.mass[i] = 0u;
        sh.count[i] = 0u;
    }
    if (threadIdx.x == 0u) {
        sh.list_bin = ~0u;
        sh.listed = 0u;
    }
    __syncthreads();
    uint32_t best = 0u;
    for (uint32_t w = 0; w < kWaves; ++w) {
        best = uint32_t(sh.of_wave[w] >> 32) > best ? uint32_t(sh.of_wave[w] >> 32) : best;
        bits = uint32_t(sh.of_wave[w]) > bits ? uint32_t(sh.of_wave[w]) : bits;
    }
    top = of_key(best);
    if (bits > 0x7F800000u || !(temperature >= 0.0f) || top == -__builtin_inff()) {
        answer(-1, 0.0f);
        return;
    }
    if (temperature == 0.0f || set.top_k == 1u) {
        find_equal(sh, row, best, 1u);
        answer(int64_t(sh.found_id), 1.0f);
        return;
    }
    if (top == __builtin_inff()) {
        // infinities share the row alone, each a mass of 1
        uint32_t mine = 0u;
        row.each([&](float l, uint32_t) __attribute__((always_inline)) { mine += l == __builtin_inff() ? 1u : 0u; });
        __syncthreads();
        added_before(mine, sh.of_wave);
        uint64_t kept = 0u;
        for (uint32_t w = 0; w < kWaves; ++w) kept += sh.of_wave[w];
        kept = set.top_k && set.top_k < kept ? set.top_k : kept;
        if (set.top_p < 1.0f) kept = wanted_of(set.top_p, kept);
        find_equal(sh, row, best, drawn_at(set.u, kept) + 1u);
        answer(int64_t(sh.found_id), float(1.0 / double(kept)));
        return;
    }
    row.top = double(top);
    row.steps = 1.4426950408889634074 * double(kSteps) / double(temperature);
    const double one = __builtin_bit_cast(double, uint64_t(1023u + p.point) << 52);
    const double least = set.min_p < 1.0f ? double(set.min_p) : 1.0;                // (not looked at where there is none)

    // Few tokens that may be kept are listed, and all else is done in the list.  top_k: as many threads' largest logits are at least the least of those that are
    // listed, so that at least top_k tokens are.  min_p alone: those that weigh enough.
    const bool by_weight = set.min_p > 0.0f && !(set.top_p < 1.0f);
    if ((set.top_k && set.top_k <= kList / 2u) || by_weight) {
        uint32_t last = kBins - 1u;
        if (set.top_k && set.top_k <= kList / 2u) {
            uint32_t bin;
            uint64_t q;
            if (row.weigh(own_top, bin, q)) atomicAdd(&sh.count[bin], 1u);
            __syncthreads();
            add_up_bins(sh);
            if (set.top_k <= sh.count[kBins]) last = bin_of(sh, [&](uint32_t i) __attribute__((always_inline)) { return uint64_t(sh.count[i]); }, set.top_k);
        }
        if (by_weight) {
            const double t = -double(kSteps) * log2(least) + 1.0;
            last = t < double(last) ? uint32_t(t) : last;
        }
        float low, high;
        row.reach_of(0u, last, low, high);
        row.each([&](float l, uint32_t id) __attribute__((always_inline)) {
            if (!(l >= low)) return;
            uint32_t bin;
            uint64_t q;
            if (!row.weigh(l, bin, q)) return;
            const uint32_t at = atomicAdd(&sh.listed, 1u);
            if (at >= kList) return;
            sh.list_key[at] = key_of(l);
            sh.list_id[at] = id;
            sh.list_q[at] = mass_of(height(bin), q);
        });
        __syncthreads();
        const uint32_t n = sh.listed;
        if (n <= kList) {
            draw_from_list(sh, set, n, p.point, least * one);
            answer(int64_t(sh.found_id), float(double(sh.found_q) / double(sh.found_sum)));
            return;
        }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i <= kBins; i += kThreads) {
            sh.mass[i] = 0u;
            sh.count[i] = 0u;
        }
        __syncthreads();
    }

    const bool counts = set.top_k != 0u;
    row.each([&](float l, uint32_t) __attribute__((always_inline)) {
        uint32_t bin;
        uint64_t q;
        if (!row.weigh(l, bin, q)) return;
        atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[bin]), q);
        if (counts) atomicAdd(&sh.count[bin], 1u);
    });
    __syncthreads();
    add_up_bins(sh);
    const auto mass_before = [&](uint32_t b) __attribute__((always_inline)) { return sh.mass[b]; };

    uint64_t kept = sh.mass[kBins];
    if (set.top_k && set.top_k < sh.count[kBins]) {
        const uint32_t b = bin_of(sh, [&](uint32_t i) __attribute__((always_inline)) { return uint64_t(sh.count[i]); }, set.top_k);
        const uint64_t wanted = set.top_k - sh.count[b];
        if (wanted == sh.count[b + 1u] - sh.count[b]) {
            kept = sh.mass[b + 1u];
        } else {
            find<DTYPE>(sh, row, b, [=](uint64_t count, uint64_t) { return count >= wanted; });
            kept = sh.mass[b] + mass_of(height(b), sh.found_sum);
            __syncthreads();
        }
    }
    // The bins in which the two other borders are: the first border counts, and where that is one bin's both have to be worked out.
    uint32_t bin_p = kBins, bin_m = kBins;
    uint64_t wanted = 0u;
    if (set.top_p < 1.0f) {
        wanted = wanted_of(set.top_p, kept);
        bin_p = bin_of(sh, mass_before, wanted);
    }
    if (set.min_p > 0.0f) {
        const double t = -double(kSteps) * log2(least);
        if (t < double(kBins) - 1.0) bin_m = uint32_t(rint(t));
    }
    if (bin_p < kBins && bin_p <= bin_m) {
        const uint64_t before = sh.mass[bin_p];
        const double high = height(bin_p);
        find<DTYPE>(sh, row, bin_p, [=](uint64_t, uint64_t sum) { return before + mass_of(high, sum) >= wanted; });
        const uint64_t upto = before + mass_of(high, sh.found_sum);
        kept = upto < kept ? upto : kept;
        __syncthreads();
    }
    if (bin_m < kBins && bin_m <= bin_p) {
        const double high = height(bin_m), border = least * one;
        float lo, hi;
        row.reach_of(bin_m, bin_m, lo, hi);
        uint64_t sum = 0u;
        row.each([&](float l, uint32_t) __attribute__((always_inline)) {
            if (!(l >= lo && l <= hi)) return;
            uint32_t bin;
            uint64_t q;
            if (row.weigh(l, bin, q) && bin == bin_m && high * double(q) >= border) sum += q;
        });
        __syncthreads();
        added_before(sum, sh.of_wave);
        sum = 0u;
        for (uint32_t i = 0; i < kWaves; ++i) sum += sh.of_wave[i];
        const uint64_t upto = sh.mass[bin_m] + mass_of(high, sum);
        kept = upto < kept ? upto : kept;
    }
    const uint64_t at = drawn_at(set.u, kept);
    const uint32_t b = bin_of(sh, mass_before, at + 1u);
    const uint64_t before = sh.mass[b];
    const double high = height(b);
    find<DTYPE>(sh, row, b, [=](uint64_t, uint64_t sum) { return before + mass_of(high, sum) > at; });
    answer(int64_t(sh.found_id), float(high * double(sh.found_q) / double(kept)));
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
    const dim3 grid(groups_across(a->rows), groups_down(a->rows));
    if (a->dtype == ANSZP_OUT_F32) hipLaunchKernelGGL(sample_kernel<ANSZP_OUT_F32>, grid, dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), p);
    else hipLaunchKernelGGL(sample_kernel<ANSZP_OUT_BF16>, grid, dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), p);
    return hipGetLastError() == hipSuccess ? ANSZP_OK : ANSZP_E_HIP;
}
