// Quantises new keys and values into the pages of the 8-bit cache (awe_kv_write).
//
// For the run of tokens of one page and head: a = max |x| over the run's finite values, s' = max(s, a * (1 / 127)) with the
// scale s that the page has (0 where the run starts the page), q = round(x / s'); where s' > s the values already in the page
// become round(q s / s').  The first 8,192 values of a run are read once (they wait in registers between the maximum and the
// rounding), the rest of a longer one twice, from L2 the second time; all are written once.
//
// The list's tokens of one page stand together, so a block finds its runs by itself: it looks at `window` neighbouring slots and
// takes the runs that begin there.  Slots that are skipped may stand between a run's tokens (a list with some of its
// tokens masked): the run goes on behind them, since two blocks that shared a page would race for its scale.
#include <algorithm>
#include <type_traits>

#include "awe_internal.h"
#include "serve_common.cuh"

namespace awe {
namespace {

using namespace serve;

constexpr int kThreads = 128;
constexpr int kMostHeld = 8;  // 16-byte pieces a thread keeps in registers between the two passes

struct WriteParams {
    const void *k, *v;
    int8_t *k_cache, *v_cache;
    float *k_scale, *v_scale;
    const int64_t* slots;
    int64_t ldk, ldv, T, n_slots;
    int heads, page_log2, dim_log2, window;
};

template <bool kBf16, bool kVec>
__device__ __forceinline__ uint4 load8(const typename Half<kBf16>::type* x) {
    if constexpr (kVec) return __ldg(reinterpret_cast<const uint4*>(x));
    else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint16_t* u = reinterpret_cast<const uint16_t*>(x) + 2 * i;
            w[i] = u[0] | ((uint32_t)u[1] << 16);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// Two unsigned maxima of 16-bit magnitudes: the patterns of finite values order like the values, and a maximum of
// kInfinity or more says that an infinity or a NaN is among them.
__device__ __forceinline__ uint32_t largest8(uint4 w, uint32_t m) {
    m = __vimax3_u16x2(m, w.x & 0x7FFF7FFFu, w.y & 0x7FFF7FFFu);
    return __vimax3_u16x2(m, w.z & 0x7FFF7FFFu, w.w & 0x7FFF7FFFu);
}
template <bool kBf16>
__device__ __forceinline__ uint32_t largest_finite8(uint4 w, uint32_t m) {
    constexpr uint32_t kInfinity = kBf16 ? 0x7F80u : 0x7C00u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t x = ((&w.x)[i >> 1] >> (16 * (i & 1))) & 0x7FFFu;
        if (x < kInfinity) m = max(m, x);
    }
    return m;
}
// round(x * inverse) for finite x, 0 for NaN, +-127 for the infinities (whatever the scale).
__device__ __forceinline__ int quantise(float x, float inverse) {
    const float y = fabsf(x) <= 3.402823466e38f ? rintf(__fmul_rn(x, inverse)) : (x > 0.0f ? 127.0f : (x < 0.0f ? -127.0f : 0.0f));
    return (int)fminf(fmaxf(y, -127.0f), 127.0f);
}
template <bool kBf16>
__device__ __forceinline__ uint2 quantise8_any(uint4 w, float inverse) {
    uint32_t q[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float2 a = Half<kBf16>::unpack((&w.x)[2 * i]), b = Half<kBf16>::unpack((&w.x)[2 * i + 1]);
        q[i] = (uint32_t)(uint8_t)quantise(a.x, inverse) | (uint32_t)(uint8_t)quantise(a.y, inverse) << 8 |
               (uint32_t)(uint8_t)quantise(b.x, inverse) << 16 | (uint32_t)(uint8_t)quantise(b.y, inverse) << 24;
    }
    return make_uint2(q[0], q[1]);
}
// The same where every value is finite, so that |x * inverse| < 127.5: adding 1.5 * 2^23 rounds to an integer, ties to
// even, whose two's complement is the low byte of the sum.
template <bool kBf16>
__device__ __forceinline__ uint2 quantise8(uint4 w, float inverse) {
    uint32_t q[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float2 a = Half<kBf16>::unpack((&w.x)[2 * i]), b = Half<kBf16>::unpack((&w.x)[2 * i + 1]);
        auto round = [&](float x) { return __float_as_uint(__fadd_rn(__fmul_rn(x, inverse), 12582912.0f)); };
        q[i] = __byte_perm(__byte_perm(round(a.x), round(a.y), 0x0040), __byte_perm(round(b.x), round(b.y), 0x0040), 0x5410);
    }
    return make_uint2(q[0], q[1]);
}
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float ratio) {
    uint32_t q = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        q |= (uint32_t)(uint8_t)(int)rintf(__fmul_rn((float)(int8_t)(w >> (8 * i)), ratio)) << (8 * i);
    return q;
}

// grid: (windows of tokens, heads, keys / values).  Seven blocks on an SM (72 registers): more loads are under way than with six, and
// nothing spills as it does with eight.  19.6 k tokens of 8 heads of 128: 30.4 us; with six 31.8.
template <bool kBf16, bool kVec>
__global__ void __launch_bounds__(kThreads, 7) kv_write_kernel(WriteParams p) {
    using T16 = typename Half<kBf16>::type;
    __shared__ uint32_t warp_max[kThreads / 32];
    constexpr uint32_t kInfinity = kBf16 ? 0x7F80u : 0x7C00u;
    const int tid = threadIdx.x, lane = tid & 31, head = blockIdx.y;
    const bool values = blockIdx.z != 0;
    const T16* x = reinterpret_cast<const T16*>(values ? p.v : p.k);
    const int64_t ldx = values ? p.ldv : p.ldk;
    int8_t* cache = values ? p.v_cache : p.k_cache;
    float* scales = values ? p.v_scale : p.k_scale;
    const int dim = 1 << p.dim_log2, page_size = 1 << p.page_log2, per_row_log2 = p.dim_log2 - 3;
    auto page_of_slot = [&](int64_t slot) -> int64_t { return slot < 0 || slot >= p.n_slots ? -1 : slot >> p.page_log2; };
    auto page_of = [&](int64_t t) { return page_of_slot(p.slots[t]); };
    // A run goes on behind at most this many skipped slots (31: so many that no gap inside 32 neighbours ends it).
    const int most_skipped = max(page_size, 31);
    // Whether none of the tokens before t that are near enough, skipped ones left out, is of this page: asked by the whole
    // warp, 32 tokens at a time.
    auto no_run_before = [&](int64_t t, int64_t page) {
        for (int64_t end = t; end > 0 && t - end <= most_skipped; end -= 32) {
            const int64_t back = end - 1 - lane, other = back >= 0 && t - 1 - back <= most_skipped ? page_of(back) : -1;
            const unsigned found = __ballot_sync(~0u, other >= 0);
            if (found) return __shfl_sync(~0u, other, __ffs(found) - 1) != page;
        }
        return true;
    };
    grid_wait();
    const int64_t t_begin = (int64_t)blockIdx.x * p.window, t_end = min(p.T, t_begin + p.window);
    unsigned begins = 0;  // of the 32 tokens from t32, those that begin a run (every warp finds out for itself)
    int64_t mine = -1;    // slot of this lane's of those
    for (int64_t t32 = t_begin, t0 = 0; t32 < t_end || begins; begins &= begins - 1) {
        while (!begins && t32 < t_end) {
            const int64_t t = t32 + lane, before = t > 0 && t < t_end ? p.slots[t - 1] : -1;
            mine = t < t_end ? p.slots[t] : -1;
            const int64_t page = page_of_slot(mine), page_before = page_of_slot(before);
            begins = __ballot_sync(~0u, page >= 0 && page_before != page);
            for (unsigned ask = __ballot_sync(~0u, page >= 0 && page_before < 0 && t > 0); ask; ask &= ask - 1) {
                const int i = __ffs(ask) - 1;
                if (!no_run_before(t32 + i, __shfl_sync(~0u, page, i))) begins &= ~(1u << i);
            }
            t32 += 32;
        }
        if (!begins) break;
        t0 = t32 - 32 + __ffs(begins) - 1;
        const int64_t slot0 = __shfl_sync(~0u, mine, __ffs(begins) - 1), page = page_of_slot(slot0);
        const int place = (int)(slot0 & (page_size - 1));
        // the run: up to the last token of the same page, whether none in it is skipped, and whether all follow place by place
        int n = 1, at = 1;
        bool dense = true, in_order = true, more_to_see = true;
        auto slot_of = [&](int64_t t) { return t < p.T ? p.slots[t] : -1; };
        auto look = [&](int64_t slot) {  // at the 32 tokens from t0 + at
            const int64_t other = page_of_slot(slot);
            const unsigned same = __ballot_sync(~0u, other == page), end = __ballot_sync(~0u, other >= 0 && other != page);
            const unsigned next = __ballot_sync(~0u, slot == slot0 + at + lane);
            const unsigned more = end ? same & ((end & -end) - 1) : same;  // those in front of the first of another page
            if (more && at + __ffs(more) - 2 - (n - 1) <= most_skipped) {
                const int last = 31 - __clz(more);
                const unsigned all = last == 31 ? ~0u : (2u << last) - 1u;
                dense = dense && n == at && more == all;
                in_order = in_order && (~next & all) == 0;
                n = at + last + 1;
            }
            at += 32;
            more_to_see = !end && at - n <= most_skipped && t0 + at < p.T;
        };
        look(slot_of(t0 + at + lane));
        while (more_to_see) {
            constexpr int kAhead = 4;  // slots that are on their way together
            int64_t ahead[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) ahead[i] = slot_of(t0 + at + 32 * i + lane);
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (more_to_see) look(ahead[i]);
        }
        in_order = in_order && dense;
        // this thread's pieces: column `col` of the rows row, row + step, ... (a power of two of pieces per row divides the block)
        const int pieces = n << per_row_log2, row = tid >> per_row_log2, col = (tid & ((1 << per_row_log2) - 1)) << 3, step = kThreads >> per_row_log2;
        const T16* first = x + (t0 + row) * ldx + (int64_t)head * dim + col;
        auto piece = [&](int j) { return first + (int64_t)j * step * ldx; };  // the j-th
        // kSkips: some of the rows are to be left out (none is held: a short form for a rare case)
        auto write = [&](auto skips) {
            constexpr bool kSkips = decltype(skips)::value;
            constexpr int kHeld = kSkips ? 0 : kMostHeld;
            auto live = [&](int j) { return tid + j * kThreads < pieces && (!kSkips || page_of(t0 + row + j * step) >= 0); };
            uint4 held[kMostHeld];
#pragma unroll
            for (int j = 0; j < kHeld; ++j)
                held[j] = live(j) ? load8<kBf16, kVec>(piece(j)) : make_uint4(0, 0, 0, 0);
            float* scale = scales + page * p.heads + head;
            const float before = place > 0 ? *scale : 0.0f;
            auto block_max = [&](uint32_t m) {
                m = __reduce_max_sync(~0u, max(m & 0xFFFFu, m >> 16));
                __syncthreads();  // whoever read warp_max before has it
                if (lane == 0) warp_max[tid >> 5] = m;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < kThreads / 32; ++w) m = max(m, warp_max[w]);
                return m;
            };
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < kHeld; ++j) top = largest8(held[j], top);
            for (int j = kHeld; tid + j * kThreads < pieces; ++j)
                if (live(j)) top = largest8(load8<kBf16, kVec>(piece(j)), top);
            top = block_max(top);
            const bool finite = top < kInfinity;
            if (!finite) {
                top = 0;
#pragma unroll
                for (int j = 0; j < kHeld; ++j) top = largest_finite8<kBf16>(held[j], top);
                for (int j = kHeld; tid + j * kThreads < pieces; ++j)
                    if (live(j)) top = largest_finite8<kBf16>(load8<kBf16, kVec>(piece(j)), top);
                top = block_max(top);
            }
            const float m = Half<kBf16>::unpack(top).x;
            const float wanted = m < 7.888609052e-31f ? 0.0f : __fmul_rn(m, 1.0f / 127.0f);  // 2^-100: its reciprocal stays finite
            const float after = fmaxf(before, wanted);
            const float inverse = after > 0.0f ? 1.0f / after : 0.0f;
            int8_t* block = cache + ((page * p.heads + head) << (p.page_log2 + p.dim_log2));
            if (after > before && place > 0) {
                const float ratio = before / after;
                uint32_t* old = reinterpret_cast<uint32_t*>(block);
                for (int i = tid; i < place << (p.dim_log2 - 2); i += kThreads) old[i] = rescale4(old[i], ratio);
            }
            int8_t* to = block + (place << p.dim_log2) + 8 * tid;  // where the places follow, the pieces do
            auto out = [&](int j) {
                if (in_order) return reinterpret_cast<uint2*>(to + 8 * kThreads * j);
                const int at = (int)(p.slots[t0 + row + j * step] & (page_size - 1));
                return reinterpret_cast<uint2*>(block + (at << p.dim_log2) + col);
            };
            auto store = [&](auto quantise_piece) {
#pragma unroll
                for (int j = 0; j < kHeld; ++j)
                    if (live(j)) *out(j) = quantise_piece(held[j]);
                for (int j = kHeld; tid + j * kThreads < pieces; ++j)
                    if (live(j)) *out(j) = quantise_piece(load8<kBf16, kVec>(piece(j)));
            };
            if (finite) store([&](uint4 w) { return quantise8<kBf16>(w, inverse); });
            else store([&](uint4 w) { return quantise8_any<kBf16>(w, inverse); });
            __syncthreads();  // every thread has read the old scale
            if (tid == 0) *scale = after;
        };
        if (dense) write(std::false_type());
        else write(std::true_type());
    }
}

}  // namespace

// Checks shared by the operators that take the cache.
awe_status_t check_kv_cache(const awe_kv_cache* c) {
    if (!c || !c->k_dev || !c->v_dev || !c->k_scale_dev || !c->v_scale_dev || c->n_pages <= 0 || c->n_heads <= 0)
        return AWE_ERR_INVALID_ARG;
    if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1))) return AWE_ERR_UNSUPPORTED;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return AWE_ERR_UNSUPPORTED;
    if (c->n_pages > INT32_MAX || c->n_heads > 65535) return AWE_ERR_UNSUPPORTED;
    if ((uintptr_t)c->k_dev % 16 || (uintptr_t)c->v_dev % 16 || (uintptr_t)c->k_scale_dev % 4 || (uintptr_t)c->v_scale_dev % 4)
        return AWE_ERR_ALIGNMENT;
    return AWE_OK;
}

}  // namespace awe

using namespace awe;
using namespace awe::serve;

extern "C" awe_status_t awe_kv_write(awe_handle_t h, const awe_kv_cache* cache, const void* k_dev, const void* v_dev,
                                     awe_float_t type, int64_t T, int64_t ldk, int64_t ldv, const int64_t* slots_dev,
                                     void* stream) {
    if (!h || T < 0) return AWE_ERR_INVALID_ARG;
    const awe_status_t s = check_kv_cache(cache);
    if (s != AWE_OK) return s;
    if ((int)type < AWE_F16 || (int)type > AWE_F32) return AWE_ERR_INVALID_ARG;
    if (!is_half_type(type)) return AWE_ERR_UNSUPPORTED;
    if (T == 0) return AWE_OK;
    const int64_t width = cache->n_heads * cache->head_dim;
    if (!k_dev || !v_dev || !slots_dev || T > INT32_MAX || (T > 1 && (ldk < width || ldv < width))) return AWE_ERR_INVALID_ARG;
    if ((uintptr_t)k_dev % 2 || (uintptr_t)v_dev % 2 || (uintptr_t)slots_dev % 8) return AWE_ERR_ALIGNMENT;
    WriteParams p = {k_dev, v_dev, cache->k_dev, cache->v_dev, cache->k_scale_dev, cache->v_scale_dev, slots_dev, ldk, ldv, T,
                     cache->n_pages * cache->page_size, (int)cache->n_heads, 4, 6, 1};
    while ((1 << p.page_log2) < cache->page_size) ++p.page_log2;
    while ((1 << p.dim_log2) < cache->head_dim) ++p.dim_log2;
    // A block looks at `window` tokens: one where that leaves few blocks (each token may start a run), up to a
    // page's where there are many (then nearly every block finds one run).
    while (p.window < cache->page_size && T / (2 * p.window) * cache->n_heads * 2 >= 16 * h->sm_count) p.window *= 2;
    const dim3 grid((unsigned)((T + p.window - 1) / p.window), (unsigned)cache->n_heads, 2);
    const bool vec = (uintptr_t)k_dev % 16 == 0 && (uintptr_t)v_dev % 16 == 0 && ldk % 8 == 0 && ldv % 8 == 0;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = type == AWE_BF16 ? (vec ? launch_early(kv_write_kernel<true, true>, grid, kThreads, 0, st, p)
                                                  : launch_early(kv_write_kernel<true, false>, grid, kThreads, 0, st, p))
                                           : (vec ? launch_early(kv_write_kernel<false, true>, grid, kThreads, 0, st, p)
                                                  : launch_early(kv_write_kernel<false, false>, grid, kThreads, 0, st, p));
    if (e != cudaSuccess) return AWE_ERR_CUDA;
    h->launches += 1;
    return AWE_OK;
}
