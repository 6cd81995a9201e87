// What a serving step needs to know of the paged cache: new pages, slots, positions and starts from the
// requests' lengths (awe_kv_plan).
//
// With have_b = ceil(cached_b / P), want_b = ceil((cached_b + new_b) / P), request b takes the entries
// [base_b, base_b + want_b - have_b) of the free list, base the exclusive sum over the requests, and its new tokens
// are those from start_b, start the exclusive sum of new.  Both sums run over at most 16,384 requests, so every
// block forms all of them for itself (8 bytes read per request, from L2 after the first block) and then fills its
// share of the outputs by binary search in shared memory: one launch, no block waits for another.
// Bound by latency below about 10^5 tokens, by the 12 bytes written per token above.
#include <algorithm>

#include "awe_internal.h"
#include "serve_common.cuh"

namespace awe {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxRequests = AWE_KV_MAX_REQUESTS;

struct PlanParams {
    const int32_t *cached, *added, *free_pages;
    int32_t* table;
    int64_t* slots;
    int32_t *positions, *q_start, *ctx_len, *counts;
    int64_t ld_table, max_tokens, n_free;
    int B, page_log2, max_pages;
};

struct Sums {
    int tokens, pages, missing, longest;
};

// Last index i in [0, n) with a[i] <= x (a[0] = 0 <= x, a ascending).
__device__ __forceinline__ int last_not_above(const int* a, int n, int x) {
    int lo = 0;
    while (n > 1) {
        const int half = n >> 1;
        if (a[lo + half] <= x) lo += half;
        n -= half;
    }
    return lo;
}

// Sums of counts stay at 2^31 - 1 where they would pass it (which is associative), so that every prefix is in order
// and no place computed from one is negative, whatever the lengths are.
__device__ __forceinline__ int add_sat(int a, int b) { return (int)min((unsigned)a + (unsigned)b, 0x7FFFFFFFu); }

__global__ void __launch_bounds__(kThreads) kv_plan_kernel(PlanParams p) {
    extern __shared__ int prefix[];
    int* start = prefix;             // B + 1: first new token of each request
    int* base = prefix + p.B + 1;    // B + 1: first entry of the free list it takes
    __shared__ Sums warp_sums[kThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int mask = (1 << p.page_log2) - 1;
    auto lengths = [&](int b, int& cached, int& added) {
        cached = max(p.cached[b], 0);
        added = max(p.added[b], 0);
    };
    auto pages_of = [&](int64_t tokens) { return (int)((tokens + mask) >> p.page_log2); };

    serve::grid_wait();
    // each thread sums a run of requests, the block sums the threads, each thread writes its run's prefix
    const int per = (p.B + kThreads - 1) / kThreads, b0 = min(p.B, tid * per), b1 = min(p.B, b0 + per);
    Sums s = {0, 0, 0, 0};
    for (int b = b0; b < b1; ++b) {
        int cached, added;
        lengths(b, cached, added);
        const int have = pages_of(cached), want = pages_of((int64_t)cached + added);
        s.tokens = add_sat(s.tokens, added);
        s.pages = add_sat(s.pages, max(min(want, p.max_pages) - have, 0));
        s.missing = add_sat(s.missing, want - have);
        s.longest = max(s.longest, add_sat(cached, added));
    }
    Sums inc = s;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int a = __shfl_up_sync(~0u, inc.tokens, d), b = __shfl_up_sync(~0u, inc.pages, d),
                  c = __shfl_up_sync(~0u, inc.missing, d), m = __shfl_up_sync(~0u, inc.longest, d);
        if (lane >= d) inc = {add_sat(inc.tokens, a), add_sat(inc.pages, b), add_sat(inc.missing, c), max(inc.longest, m)};
    }
    if (lane == 31) warp_sums[warp] = inc;
    int tokens = __shfl_up_sync(~0u, inc.tokens, 1), pages = __shfl_up_sync(~0u, inc.pages, 1);  // of the lanes before
    if (lane == 0) tokens = pages = 0;
    __syncthreads();
    Sums total = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        const Sums o = warp_sums[w];
        if (w < warp) tokens = add_sat(tokens, o.tokens), pages = add_sat(pages, o.pages);
        total = {add_sat(total.tokens, o.tokens), add_sat(total.pages, o.pages), add_sat(total.missing, o.missing), max(total.longest, o.longest)};
    }
    for (int b = b0; b < b1; ++b) {
        int cached, added;
        lengths(b, cached, added);
        start[b] = tokens;
        base[b] = pages;
        if (blockIdx.x == 0) {
            p.q_start[b] = tokens;
            p.ctx_len[b] = add_sat(cached, added);
        }
        tokens = add_sat(tokens, added);
        pages = add_sat(pages, max(min(pages_of((int64_t)cached + added), p.max_pages) - pages_of(cached), 0));
    }
    if (tid == 0) {
        start[p.B] = total.tokens;
        base[p.B] = total.pages;
        if (blockIdx.x == 0) {
            const int taken = (int)min((int64_t)total.pages, p.n_free);
            p.q_start[p.B] = total.tokens;
            p.counts[0] = taken;
            p.counts[1] = total.tokens;
            p.counts[2] = total.missing - taken;
            p.counts[3] = total.longest;
        }
    }
    __syncthreads();

    const int64_t first = (int64_t)blockIdx.x * kThreads + tid, step = (int64_t)gridDim.x * kThreads;
    for (int64_t i = first; i < total.pages; i += step) {
        const int b = last_not_above(base, p.B, (int)i);
        const int j = pages_of(max(p.cached[b], 0)) + (int)i - base[b];
        if (j < p.max_pages) p.table[b * p.ld_table + j] = i < p.n_free ? p.free_pages[i] : -1;
    }
    for (int64_t t = first; t < p.max_tokens; t += step) {
        int64_t slot = -1;
        int pos = -1;
        if (t < total.tokens) {
            const int b = last_not_above(start, p.B, (int)t);
            const int cached = max(p.cached[b], 0);
            const unsigned at = (unsigned)cached + (unsigned)((int)t - start[b]);  // below 2^32
            pos = (int)min(at, 0x7FFFFFFFu);
            const int j = (int)(at >> p.page_log2), have = pages_of(cached);
            int page = -1;
            if (j < p.max_pages) {
                const int64_t i = (int64_t)base[b] + j - have;
                page = j < have ? p.table[b * p.ld_table + j] : (i < p.n_free ? p.free_pages[i] : -1);
            }
            if (page >= 0) slot = ((int64_t)page << p.page_log2) + (at & mask);
        }
        p.slots[t] = slot;
        if (p.positions) p.positions[t] = pos;
    }
}

// Whether two arrays of n and m elements share memory.
bool overlap(const int32_t* a, int64_t n, const int32_t* b, int64_t m) {
    return n > 0 && m > 0 && (uintptr_t)a < (uintptr_t)(b + m) && (uintptr_t)b < (uintptr_t)(a + n);
}

}  // namespace
}  // namespace awe

using namespace awe;

extern "C" awe_status_t awe_kv_plan(awe_handle_t h, const int32_t* cached_len_dev, const int32_t* new_len_dev, int64_t B,
                                    int64_t page_size, const int32_t* free_pages_dev, int64_t n_free,
                                    int32_t* block_table_dev, int64_t max_pages, int64_t ld_table, int64_t* slots_dev,
                                    int32_t* positions_dev, int64_t max_tokens, int32_t* q_start_dev,
                                    int32_t* ctx_len_dev, int32_t* counts_dev, void* stream) {
    if (!h || !q_start_dev || !counts_dev || B < 0 || n_free < 0 || max_tokens < 0 || max_tokens > INT32_MAX ||
        n_free > INT32_MAX || max_pages <= 0 || max_pages > INT32_MAX || ld_table < max_pages)
        return AWE_ERR_INVALID_ARG;
    if (B > 0 && (!cached_len_dev || !new_len_dev || !block_table_dev || !ctx_len_dev)) return AWE_ERR_INVALID_ARG;
    if ((n_free > 0 && !free_pages_dev) || (max_tokens > 0 && !slots_dev)) return AWE_ERR_INVALID_ARG;
    if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1)) || B > kMaxRequests) return AWE_ERR_UNSUPPORTED;
    if ((uintptr_t)cached_len_dev % 4 || (uintptr_t)new_len_dev % 4 || (uintptr_t)free_pages_dev % 4 ||
        (uintptr_t)block_table_dev % 4 || (uintptr_t)slots_dev % 8 || (uintptr_t)positions_dev % 4 ||
        (uintptr_t)q_start_dev % 4 || (uintptr_t)ctx_len_dev % 4 || (uintptr_t)counts_dev % 4)
        return AWE_ERR_ALIGNMENT;
    // Every block reads the lengths for itself, at a time of its own: what one of them writes must not lie there.
    for (const int32_t* lengths : {cached_len_dev, new_len_dev})
        if (overlap(lengths, B, ctx_len_dev, B) || overlap(lengths, B, q_start_dev, B + 1) || overlap(lengths, B, counts_dev, 4)) return AWE_ERR_INVALID_ARG;
    int page_log2 = 4;
    while ((1 << page_log2) < page_size) ++page_log2;
    PlanParams p = {cached_len_dev, new_len_dev, free_pages_dev, block_table_dev, slots_dev,       positions_dev,
                    q_start_dev,    ctx_len_dev, counts_dev,     ld_table,        max_tokens,      n_free,
                    (int)B,         page_log2,   (int)max_pages};
    // The limit is the kernel's, not this launch's: raised to the most, so that no other thread's call finds it lower than its own.
    const size_t smem = 2 * (size_t)(B + 1) * sizeof(int);
    static std::atomic<uint64_t> done{0};
    if (serve::allow_smem(kv_plan_kernel, 2 * (kMaxRequests + 1) * (int)sizeof(int), h->device, done) != cudaSuccess) return AWE_ERR_CUDA;
    const int64_t items = std::max(max_tokens, B);
    const int blocks = (int)std::max<int64_t>(1, std::min<int64_t>((items + kThreads - 1) / kThreads, 4 * h->sm_count));
    if (serve::launch_early(kv_plan_kernel, dim3(blocks), kThreads, smem, (cudaStream_t)stream, p) != cudaSuccess) return AWE_ERR_CUDA;
    h->launches += 1;
    return AWE_OK;
}
