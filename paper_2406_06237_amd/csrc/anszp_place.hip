// New tokens placed in a paged cache, for gfx950: what a step's page tables, lengths, starts and slots are, from how many tokens each sequence
// holds and gets, without the host.  With P tokens a page and the free pages as a stack:
//   old[s]  = 0 where the sequence ends (its ceil(lengths[s] / P) pages go on the stack, sequence by sequence), else lengths[s]
//   need[s] = ceil((old[s] + new[s]) / P) - ceil(old[s] / P)      upto[s] = need[0] + ... + need[s]
//   the j-th page that s gets is stack[top - 1 - (upto[s] - need[s] + j)], if upto[s] <= top; else s gets nothing
//   slot    = page * P + position mod P
// All of it are sums over the sequences and a look-up a token, so nothing depends on the order in which threads arrive.
//
// One workgroup adds up over the sequences and leaves a record for each; a thread a token then finds its sequence in the starts and its page
// in the table or on the stack, and writes the table where it is the first in its page.  Latency bounds it, of loads and of the sums' barriers: 16 sequences with a
// token each take 3.6 us, 512 sequences with 151000 tokens and some of them ended 7.0 for the sums, 2.5 for the pages that go back and 4.6 for the tokens, whose
// starts, looked up eight or nine times each, are in LDS (from memory 7).
#include <hip/hip_runtime.h>

#include "anszp_numbers.h"

namespace {

// What a sequence's tokens need to know: tokens before this step (-1: refused), pages before it, and the stack's place of its first new page; and
// where its pages go that it gives back, and how many.
struct Record {
    int32_t old, pages, top, back_at, back;
};

struct PlaceParams {
    int32_t* pages;
    const int32_t* lengths;
    int32_t* lengths_out;
    const int32_t* fresh;
    const int32_t* ends;
    int32_t* free;
    const int32_t* n_free;
    int32_t* n_free_out;
    int64_t* slots;
    int32_t* owners;
    int32_t* starts;
    uint32_t* status;
    int32_t* last;
    Record* records;
    uint32_t n_seqs, n_tokens, free_room, width, page_log;
};

constexpr uint32_t kInLds = 2048;       // sequences whose starts a workgroup keeps

__device__ __forceinline__ void tell(const PlaceParams& p) {
    if (p.status) {
        atomicOr(&p.status[0], ANSZP_ST_BAD_DESC);
        atomicAdd(&p.status[1], 1u);
    }
}

// The sum of `v` over the threads before this one, and over all.
struct Sums {
    int64_t before, all;
};
template <uint32_t THREADS>
__device__ __forceinline__ Sums added_up(int64_t v) {
    constexpr uint32_t kWaves = THREADS / 64u;
    __shared__ int64_t of_wave[kWaves];
    int64_t upto = v;
    for (uint32_t d = 1; d < 64u; d <<= 1) {
        const int64_t other = __shfl_up(upto, d);
        if ((threadIdx.x & 63u) >= d) upto += other;
    }
    if ((threadIdx.x & 63u) == 63u) of_wave[threadIdx.x >> 6] = upto;
    __syncthreads();
    Sums r = {upto - v, 0};
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w) {
        const int64_t other = of_wave[w];
        r.before += w < threadIdx.x >> 6 ? other : 0;
        r.all += other;
    }
    __syncthreads();
    return r;
}

// The last of n rising numbers that is no larger than `v` (the first one is).
template <class T>
__device__ __forceinline__ uint32_t last_not_above(const T* rising, uint32_t n, T v) {
    uint32_t lo = 0u, hi = n;
    while (hi - lo > 1u) {
        const uint32_t mid = lo + (hi - lo) / 2u;
        if (rising[mid] <= v) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ uint32_t pages_for(int64_t tokens, uint32_t page_log) { return uint32_t((tokens + (1ll << page_log) - 1) >> page_log); }

__device__ __forceinline__ void place_token(const PlaceParams& p, const int32_t* starts, const Record* records, uint32_t t) {
    int64_t slot = -1;
    int32_t owner = -1;
    if (int32_t(t) < starts[p.n_seqs]) {
        // (sequences without new tokens begin where the next one does: the last one that begins here has the token)
        const uint32_t s = last_not_above(starts, p.n_seqs, int32_t(t));
        const Record r = records[s];
        owner = int32_t(s);
        if (r.old >= 0) {
            const uint32_t at = uint32_t(r.old) + t - uint32_t(starts[s]), column = at >> p.page_log, inside = at & ((1u << p.page_log) - 1u);
            const uint64_t entry = uint64_t(s) * p.width + column;
            int32_t page;
            if (column < uint32_t(r.pages)) {
                page = p.pages[entry];
            } else {
                page = p.free[uint32_t(r.top) - (column - uint32_t(r.pages))];
                if (inside == 0u) p.pages[entry] = page;
            }
            if (page >= 0) slot = (int64_t(page) << p.page_log) + inside;
            else tell(p);
        }
    }
    p.slots[t] = slot;
    if (p.owners) p.owners[t] = owner;
}

// Sums over the sequences; ALONE: the pages that go back and the tokens' places as well, with what they need in LDS where there is a thread for each sequence.
template <uint32_t THREADS, bool ALONE>
__global__ __launch_bounds__(THREADS) void place_sequences_kernel(PlaceParams p) {
    __shared__ int32_t first_of[THREADS], starts[THREADS + 1u];
    __shared__ Record records[THREADS];
    const int64_t room = int64_t(p.width) << p.page_log;
    const bool one_each = ALONE && p.n_seqs <= THREADS;
    int64_t top = p.n_free[0];
    if (top < 0 || top > p.free_room) {
        top = top < 0 ? 0 : p.free_room;
        if (threadIdx.x == 0u) tell(p);
    }
    if (p.ends) {
        for (uint32_t from = 0; from < p.n_seqs; from += THREADS) {
            const uint32_t s = from + threadIdx.x;
            uint32_t back = 0u;
            if (s < p.n_seqs && p.ends[s]) {
                const int64_t held = p.lengths[s];
                if (held < 0 || held > room) tell(p);
                back = pages_for(held < 0 ? 0 : held > room ? room : held, p.page_log);
            }
            const Sums sums = added_up<THREADS>(back);
            // (a stack that its own pages overflow holds some twice; what is beyond its room is lost, and told)
            const int64_t fits = sums.all <= int64_t(p.free_room) - top ? sums.all : int64_t(p.free_room) - top;
            if (fits < sums.all && threadIdx.x == 0u) tell(p);
            const int64_t first = sums.before < fits ? sums.before : fits;
            if constexpr (ALONE) {
                // The pages that go back are shared out to the threads, whichever sequences they are of.
                first_of[threadIdx.x] = int32_t(first);
                __syncthreads();
                for (int64_t j = threadIdx.x; j < fits; j += THREADS) {
                    const uint32_t i = last_not_above(first_of, THREADS, int32_t(j));
                    p.free[top + j] = p.pages[uint64_t(from + i) * p.width + uint32_t(j - first_of[i])];
                }
                __syncthreads();
            } else if (s < p.n_seqs) {
                p.records[s].back_at = int32_t(top + first);
                p.records[s].back = int32_t(first + back < fits ? back : fits - first);
            }
            top += fits;
        }
    }
    int64_t tokens = 0, pages = 0, taken = 0;
    for (uint32_t from = 0; from < p.n_seqs; from += THREADS) {
        const uint32_t s = from + threadIdx.x;
        const bool there = s < p.n_seqs;
        const int32_t held = there ? p.lengths[s] : 0, fresh = there ? p.fresh[s] : 0;
        const bool ended = there && p.ends && p.ends[s];
        const int64_t old = ended ? 0 : held, more = fresh < 0 ? 0 : fresh;
        const Sums t = added_up<THREADS>(more);
        const int64_t start = tokens + t.before;
        tokens += t.all;
        bool served = fresh >= 0 && old >= 0 && old + more <= room && start + more <= p.n_tokens;
        const uint32_t have = served ? pages_for(old, p.page_log) : 0u, need = served ? pages_for(old + more, p.page_log) - have : 0u;
        const Sums n = added_up<THREADS>(need);
        const int64_t upto = pages + n.before + need;
        pages += n.all;
        served = served && (need == 0u || upto <= top);
        // (what is served lies in front of all that is not, so the last one's sum is what has been taken)
        int64_t last = served && need ? upto : 0;
        for (uint32_t d = 32; d; d >>= 1) {
            const int64_t other = __shfl_xor(last, d);
            last = other > last ? other : last;
        }
        __shared__ int64_t lasts[THREADS / 64u];
        if ((threadIdx.x & 63u) == 0u) lasts[threadIdx.x >> 6] = last;
        __syncthreads();
#pragma unroll
        for (uint32_t w = 0; w < THREADS / 64u; ++w) taken = lasts[w] > taken ? lasts[w] : taken;
        if (there) {
            if (!served) tell(p);
            const int32_t at = int32_t(start < p.n_tokens ? start : p.n_tokens);
            const Record r = {served ? int32_t(old) : -1, int32_t(have), int32_t(top - 1 - (upto - need)), 0, 0};
            if (one_each) {
                records[threadIdx.x] = r;
                starts[threadIdx.x] = at;
            } else {
                p.records[s].old = r.old;
                p.records[s].pages = r.pages;
                p.records[s].top = r.top;
            }
            p.starts[s] = at;
            p.lengths_out[s] = int32_t(served ? old + more : old);
            if (p.last) p.last[s] = served && more ? int32_t(start + more - 1) : -1;
        }
    }
    __syncthreads();                                                // (n_free may be its own output)
    if (threadIdx.x == 0u) {
        const int32_t all = int32_t(tokens < p.n_tokens ? tokens : p.n_tokens);
        if (one_each) starts[p.n_seqs] = all;
        p.starts[p.n_seqs] = all;
        p.n_free_out[0] = int32_t(top - taken);
    }
    if constexpr (ALONE) {
        __syncthreads();
        for (uint32_t t = threadIdx.x; t < p.n_tokens; t += THREADS) {
            if (one_each) place_token(p, starts, records, t);
            else place_token(p, p.starts, p.records, t);
        }
    }
}

// The pages that go back, a workgroup for each sequence.
__global__ __launch_bounds__(256) void place_back_kernel(PlaceParams p) {
    for (uint32_t s = blockIdx.x; s < p.n_seqs; s += gridDim.x) {
        const Record r = p.records[s];
        for (uint32_t j = threadIdx.x; int32_t(j) < r.back; j += 256u) p.free[uint32_t(r.back_at) + j] = p.pages[uint64_t(s) * p.width + j];
    }
}

__global__ __launch_bounds__(256) void place_tokens_kernel(PlaceParams p) {
    __shared__ int32_t starts[kInLds + 1u];
    const uint64_t t = uint64_t(blockIdx.x) * 256u + threadIdx.x;
    if (p.n_seqs <= kInLds) {
        for (uint32_t s = threadIdx.x; s <= p.n_seqs; s += 256u) starts[s] = p.starts[s];
        __syncthreads();
        if (t < p.n_tokens) place_token(p, starts, p.records, uint32_t(t));
    } else if (t < p.n_tokens) {
        place_token(p, p.starts, p.records, uint32_t(t));
    }
}

// The threads of the one workgroup that does all of a call, or 0: it has few tokens to place and few sequences whose pages could go back.  (16 sequences with a token
// each: 3.6 us in one launch, 5.3 and 1.8 in two.)  256 keep what the tokens need in LDS.
uint32_t alone(const anszp_place_args_t& a) {
    return a.n_tokens <= 1024u && a.n_seqs <= 256u && !a.ends ? 256u : a.n_tokens <= 4096u && (!a.ends || a.n_seqs <= 64u) ? 1024u : 0u;
}

int place_check(const anszp_place_args_t& a) {
    if (a.page_size < 16u || a.page_size > 65536u || (a.page_size & (a.page_size - 1u)) || a.table_width == 0u || a.n_seqs >= 1ull << 24 || a.n_tokens >= 1ull << 31 ||
        a.free_room >= 1ull << 31 || uint64_t(a.table_width) * a.page_size > 1ull << 30)
        return ANSZP_E_RANGE;
    return ANSZP_OK;
}

}  // namespace

extern "C" uint64_t anszp_place_workspace_bytes(const anszp_place_args_t* a) {
    return !a || place_check(*a) || alone(*a) == 256u ? 0u : (a->n_seqs * sizeof(Record) + 15u) & ~15ull;
}

extern "C" int anszp_place(const anszp_place_args_t* a, void* hip_stream) {
    if (!a) return ANSZP_E_NULL;
    const int rc = place_check(*a);
    if (rc) return rc;
    if (!a->n_free || !a->n_free_out || !a->starts || (a->n_tokens && !a->slots) || (a->free_room && !a->free_pages)) return ANSZP_E_NULL;
    const uint64_t need = anszp_place_workspace_bytes(a);
    if ((a->n_seqs && (!a->pages || !a->lengths || !a->lengths_out || !a->new_tokens)) || (need && !a->workspace)) return ANSZP_E_NULL;
    if (a->workspace_bytes < need || (reinterpret_cast<uintptr_t>(a->workspace) & 15u)) return ANSZP_E_RANGE;
    // What is written may meet nothing that other threads still read or write: lengths and n_free may be their own outputs.
    const Rows written[] = {{a->pages, 1, 0, a->n_seqs * a->table_width * 4u}, {a->free_pages, 1, 0, a->free_room * 4u}, {a->slots, 1, 0, a->n_tokens * 8u},
                            {a->owners, 1, 0, a->n_tokens * 4u}, {a->starts, 1, 0, (a->n_seqs + 1u) * 4u}, {a->workspace, 1, 0, need},
                            {a->lengths_out, 1, 0, a->n_seqs * 4u}, {a->n_free_out, 1, 0, 4}, {a->last, 1, 0, a->n_seqs * 4u}};
    const Rows lengths = {a->lengths, 1, 0, a->n_seqs * 4u}, n_free = {a->n_free, 1, 0, 4};
    const Rows read[] = {{a->new_tokens, 1, 0, a->n_seqs * 4u}, {a->ends, 1, 0, a->n_seqs * 4u}};
    for (uint32_t i = 0; i < 9u; ++i) {
        if (written[i].width == 0u) continue;
        for (uint32_t j = 0; j < i; ++j)
            if (written[j].width && meet(written[i], written[j])) return ANSZP_E_RANGE;
        for (const Rows& r : read)
            if (r.width && meet(written[i], r)) return ANSZP_E_RANGE;
        if (lengths.width && (i == 6u ? meet_elsewhere(written[i], lengths) : meet(written[i], lengths))) return ANSZP_E_RANGE;
        if (i == 7u ? meet_elsewhere(written[i], n_free) : meet(written[i], n_free)) return ANSZP_E_RANGE;
    }
    PlaceParams p = {a->pages, a->lengths, a->lengths_out, a->new_tokens, a->ends, a->free_pages, a->n_free, a->n_free_out, a->slots, a->owners, a->starts, a->status, a->last,
                     static_cast<Record*>(a->workspace), static_cast<uint32_t>(a->n_seqs), static_cast<uint32_t>(a->n_tokens), static_cast<uint32_t>(a->free_room),
                     a->table_width, static_cast<uint32_t>(__builtin_ctz(a->page_size))};
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (alone(*a) == 256u) {
        hipLaunchKernelGGL((place_sequences_kernel<256u, true>), dim3(1), dim3(256), 0, s, p);
    } else if (alone(*a) == 1024u) {
        hipLaunchKernelGGL((place_sequences_kernel<1024u, true>), dim3(1), dim3(1024), 0, s, p);
    } else {
        hipLaunchKernelGGL((place_sequences_kernel<1024u, false>), dim3(1), dim3(1024), 0, s, p);
        if (a->ends && a->n_seqs) hipLaunchKernelGGL(place_back_kernel, dim3(static_cast<uint32_t>(a->n_seqs < 65536u ? a->n_seqs : 65536u)), dim3(256), 0, s, p);
        if (a->n_tokens) hipLaunchKernelGGL(place_tokens_kernel, dim3(static_cast<uint32_t>((a->n_tokens + 255u) / 256u)), dim3(256), 0, s, p);
    }
    return hipGetLastError() == hipSuccess ? ANSZP_OK : ANSZP_E_HIP;
}
