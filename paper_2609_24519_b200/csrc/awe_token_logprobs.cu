// Log probabilities of given tokens, entropy and the most likely tokens of rows of logits (awe_token_logprobs).
//
// With M the largest logit of a row and c = scale / ln 2:   t_j = (x_j - M) c,   S0 = sum 2^t_j,   S1 = sum 2^t_j t_j,
//   z = ln S0:   lse = scale M + z,   log p_j = scale (x_j - M) - z,   entropy = z - ln 2 S1 / S0.
// M is subtracted first: a product x c could pass FP32 where logits are a type's lowest value.
// One pass: every thread keeps a maximum of its own and rescales its two sums when it grows.
//
// The most likely tokens.  The top_k-th largest of a block's 256 thread maxima is a bound that top_k elements reach, and few others do:
// the threads whose maximum reaches it have their elements looked at again (in the cache) by their warp, which gathers those that do, some 22 for
// 20; each of them finds its place by counting the ones before it.  Blocks' lists are joined in pairs: of two lists in order, the larger of a[i]
// and b[31 - i] are the best 32, in an order that five exchanges sort.  Where more reach the bound than there is room for (constrained rows, of
// which few tokens are not masked, or equal logits: a warp all of whose threads reach it says so without looking), what lies above the bound is
// gathered, and then the lowest tokens at the bound, found by a count in the tokens' order, which ends where there are enough.  Where too many lie
// above it (with few threads), the top_k-th largest of those that found room is a larger bound, and so on.  128 rows of 131,072 (BF16), 10
// tokens left and 20 alternatives: 19 us (each element gathered and then inserted into a list: 105).  (A looser bound from each warp's
// maxima alone saves the joining of eight lists, but gathers more: 17.5 -> 23 us.)
//
// HBM bounds many rows; a single row is spread over a cluster of blocks that join in shared memory, which bounds it by latency.
// 2,048 rows of 50,257 (FP16): 44 us = 4.7 TB/s, with 77 % of the issue slots and 61 % of the exponentials' rate; 128 rows of 131,072 (BF16) with 20
// alternatives 17.5 us, without 10.7; one row of 32,000 (FP32) 7.0 us.
#include <cooperative_groups.h>

#include <algorithm>

#include "awe_internal.h"
#include "serve_common.cuh"

namespace cg = cooperative_groups;

namespace awe {
namespace {

using namespace serve;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kPieces = 4;  // 16-byte pieces a thread has on their way
constexpr int kMostCluster = 8;
constexpr int kNoToken = 0x7FFFFFFF;
constexpr float kLn2 = 0.693147180559945f;

struct LogprobParams {
    const void* logits;
    const int32_t* tokens;
    float *logprob, *entropy, *lse, *top_logprob;
    int32_t* top_id;
    int64_t ld;
    float scale;
    int V, top;
};

// A token and its logit; `before` is the order of the answer: larger first, then the lower token.
struct Entry {
    float x;
    int id;
};
__device__ __forceinline__ bool before(const Entry& a, const Entry& b) { return a.x > b.x || (a.x == b.x && a.id < b.id); }
__device__ __forceinline__ Entry from_lane(const Entry& a, int lane) { return {__shfl_sync(~0u, a.x, lane), __shfl_sync(~0u, a.id, lane)}; }
// The best 32 of two lists in order, in order; `other_reversed` is the second from its end.
__device__ __forceinline__ Entry join_lists(Entry mine, const Entry& other_reversed, int lane) {
    if (before(other_reversed, mine)) mine = other_reversed;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        const Entry o = {__shfl_xor_sync(~0u, mine.x, d), __shfl_xor_sync(~0u, mine.id, d)};
        if (before(o, mine) == !(lane & d)) mine = o;
    }
    return mine;
}

__device__ __forceinline__ float max_nan(float a, float b) {
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}

template <int kType>
struct Piece {  // 16 bytes of logits
    static constexpr int kCount = kType == AWE_F32 ? 4 : 8;
    using T = typename std::conditional<kType == AWE_F32, float, uint16_t>::type;
    static __device__ __forceinline__ float one(const T* x) {
        if constexpr (kType == AWE_F32) return *x;
        else return Half<kType == AWE_BF16>::unpack(*x).x;
    }
    static __device__ __forceinline__ float at(const uint4& w, int i) {
        if constexpr (kType == AWE_F32) return __uint_as_float((&w.x)[i]);
        else {
            const float2 f = Half<kType == AWE_BF16>::unpack((&w.x)[i >> 1]);
            return i & 1 ? f.y : f.x;
        }
    }
    // The same of an element that is not known beforehand.
    static __device__ __forceinline__ float pick(const uint4& w, int i) {
        const int word = kType == AWE_F32 ? i : i >> 1;
        const uint32_t low = word & 1 ? w.y : w.x, high = word & 1 ? w.w : w.z, x = word & 2 ? high : low;
        if constexpr (kType == AWE_F32) return __uint_as_float(x);
        else return Half<kType == AWE_BF16>::unpack(i & 1 ? x >> 16 : x).x;
    }
    // Masked tokens alone, and a first element with nothing behind it.
    static __device__ __forceinline__ uint4 nothing() {
        constexpr uint32_t kMasked = kType == AWE_F32 ? 0xFF800000u : (kType == AWE_BF16 ? 0xFF80FF80u : 0xFC00FC00u);
        return make_uint4(kMasked, kMasked, kMasked, kMasked);
    }
    static __device__ __forceinline__ uint4 single(float x) {
        if constexpr (kType == AWE_F32) return make_uint4(__float_as_uint(x), 0, 0, 0);
        else return make_uint4(Half<kType == AWE_BF16>::pack(x, 0.0f), 0, 0, 0);
    }
    // The largest; NaN if one is.
    static __device__ __forceinline__ float largest(const uint4& w) {
        if constexpr (kType == AWE_F32)
            return max_nan(max_nan(__uint_as_float(w.x), __uint_as_float(w.y)), max_nan(__uint_as_float(w.z), __uint_as_float(w.w)));
        else if constexpr (kType == AWE_BF16) {
            auto b = [](uint32_t x) { return *reinterpret_cast<const __nv_bfloat162*>(&x); };
            const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(b(w.x), b(w.y)), __hmax2_nan(b(w.z), b(w.w)));
            return __bfloat162float(__hmax_nan(m.x, m.y));
        } else {
            auto b = [](uint32_t x) { return *reinterpret_cast<const __half2*>(&x); };
            const __half2 m = __hmax2_nan(__hmax2_nan(b(w.x), b(w.y)), __hmax2_nan(b(w.z), b(w.w)));
            return __half2float(__hmax_nan(m.x, m.y));
        }
    }
};

struct Sums {
    float m, s0, s1;  // maximum (NaN once a NaN was seen), S0 and S1 against it
};
// Brings sums to a larger maximum: t becomes t - g.
__device__ __forceinline__ void raise(Sums& s, float m, float c) {
    if (s.s0 != 0.0f) {
        const float g = (m - s.m) * c, a = exp2_approx(-g);
        s.s1 = a == 0.0f ? 0.0f : fmaf(-g, s.s0, s.s1) * a;
        s.s0 *= a;
    }
    s.m = m;
}
__device__ __forceinline__ Sums join_sums(Sums a, Sums b, float c) {
    const float m = max_nan(a.m, b.m);
    raise(a, m, c);
    raise(b, m, c);
    return {m, a.s0 + b.s0, a.s1 + b.s1};
}

constexpr int kRoom = kThreads;  // for gathered elements
struct Shared {
    Sums sums[kWarps];
    Entry list[kWarps][32];
    Entry found[kRoom];  // gathered elements
    int gathered;
    float maxima[kWarps][32];
    int most[kWarps];
    Sums block_sums;
    Entry block_list[32];
    int bound;  // as an ordered whole number
};
__device__ __forceinline__ int ordered(float x) {
    const int b = __float_as_int(x);
    return b < 0 ? b ^ 0x7FFFFFFF : b;
}
__device__ __forceinline__ float from_ordered(int b) { return __int_as_float(b < 0 ? b ^ 0x7FFFFFFF : b); }

// grid: a cluster for each row.
template <int kType, bool kTop>
__global__ void __launch_bounds__(kThreads) token_logprobs_kernel(const LogprobParams p) {
    using P = Piece<kType>;
    using T = typename P::T;
    __shared__ Shared sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int parts = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t row = blockIdx.x / parts;
    const float c = p.scale * 1.44269504088896f;
    if constexpr (kTop) {
        sh.found[tid] = {-INFINITY, kNoToken};
    }
    __syncthreads();
    grid_wait();
    const T* x = reinterpret_cast<const T*>(p.logits) + row * p.ld;
    // whole 16-byte pieces lie between `head` and `tail` elements at the ends of the row
    const int head = min(p.V, (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T)), pieces = (p.V - head) / P::kCount;
    const int tail_at = head + pieces * P::kCount;
    const int begin = (int)((int64_t)pieces * rank / parts), end = (int)((int64_t)pieces * (rank + 1) / parts);
    const uint4* from = reinterpret_cast<const uint4*>(x + head);

    // the given token's logit is on its way meanwhile
    int token = -1;
    float given = 0.0f;
    if (p.logprob && rank == 0 && tid == 0) {
        token = p.tokens[row];
        if (token >= 0 && token < p.V) given = P::one(x + token);
    }

    Sums own = {-INFINITY, 0.0f, 0.0f};
    Entry best = {-INFINITY, kNoToken};  // this lane's of the list
    auto add = [&](const uint4& w, int count) {
        const float m = own.m == -INFINITY ? 0.0f : own.m;
#pragma unroll
        for (int i = 0; i < P::kCount; ++i) {
            if (i >= count) continue;
            const float t = fmaxf((P::at(w, i) - m) * c, -200.0f);  // of a masked token: its exponential is 0
            const float e = exp2_approx(t);
            own.s0 += e;
            own.s1 = fmaf(e, t, own.s1);
        }
    };
    // the ends of the row, an element a thread, by the first warp of the first block and the last of the last: f(element, its place)
    auto at_ends = [&](auto f) {
        if (rank == 0 && warp == 0 && lane < head) f(P::one(x + lane), lane);
        if (rank == parts - 1 && warp == kWarps - 1 && lane < p.V - tail_at) f(P::one(x + tail_at + lane), tail_at + lane);
    };
    uint4 w[kPieces];
    for (int i0 = begin + tid; i0 < end; i0 += kThreads * kPieces) {
        float most = -INFINITY;
#pragma unroll
        for (int u = 0; u < kPieces; ++u) {
            const int i = i0 + u * kThreads;
            w[u] = P::nothing();
            if (i < end) w[u] = __ldg(from + i);
        }
#pragma unroll
        for (int u = 0; u < kPieces; ++u) most = max_nan(most, P::largest(w[u]));
        if (!(most <= own.m)) raise(own, max_nan(own.m, most), c);
#pragma unroll
        for (int u = 0; u < kPieces; ++u) add(w[u], P::kCount);
    }
    at_ends([&](float one, int) {
        const float m = max_nan(own.m, one);
        if (m != own.m) raise(own, m, c);
        add(P::single(one), 1);
    });

    // ---- sums against the block's maximum, as whole numbers in order (NaN above all)
    const int warp_most = __reduce_max_sync(~0u, own.m == own.m ? ordered(own.m) : 0x7FFFFFFF);
    if (lane == 0) sh.most[warp] = warp_most;
    if (tid == 0) sh.gathered = 0;
    __syncthreads();
    int most_of_block = sh.most[0];
#pragma unroll
    for (int i = 1; i < kWarps; ++i) most_of_block = max(most_of_block, sh.most[i]);
    const float thread_most = own.m == own.m ? own.m : -INFINITY;  // of a thread with a NaN it is not known
    const float asked_most = own.m == own.m ? own.m : INFINITY;  // its elements are looked at
    raise(own, from_ordered(most_of_block), c);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) own.s0 += __shfl_xor_sync(~0u, own.s0, d), own.s1 += __shfl_xor_sync(~0u, own.s1, d);
    if (lane == 0) sh.sums[warp] = own;

    if constexpr (kTop) {
        // ---- the bound: the top_k-th largest of the thread maxima
        float m = thread_most;
        if (p.top > 1) {
#pragma unroll
            for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
                for (int d = k >> 1; d > 0; d >>= 1) {
                    const float o = __shfl_xor_sync(~0u, m, d);
                    m = ((lane & d) == 0) == ((lane & k) == 0) ? fmaxf(m, o) : fminf(m, o);
                }
            sh.maxima[warp][lane] = m;
            __syncthreads();
            for (int step = 1; step < kWarps; step <<= 1) {
                if (warp % (2 * step) == 0) {
                    m = fmaxf(m, sh.maxima[warp + step][31 - lane]);
#pragma unroll
                    for (int d = 16; d > 0; d >>= 1) {
                        const float o = __shfl_xor_sync(~0u, m, d);
                        m = lane & d ? fminf(m, o) : fmaxf(m, o);
                    }
                    sh.maxima[warp][lane] = m;
                }
                __syncthreads();
            }
        }
        // of one alternative it is the block's maximum, beside a NaN that of the threads that have none
        if (p.top == 1) {
            m = from_ordered(most_of_block);
            if (most_of_block == 0x7FFFFFFF) {
                if (tid == 0) sh.bound = ordered(-INFINITY);
                __syncthreads();
                atomicMax(&sh.bound, ordered(thread_most));
                __syncthreads();
                m = from_ordered(sh.bound);
            }
        }
        float least = p.top > 1 ? sh.maxima[0][p.top - 1] : m;
        int gathered;
        for (bool above = false;; above = true) {
            // ---- what is `least` or more
            auto gather = [&](float logit, int id) {
                if (!(logit >= least)) return;
                const int at = atomicAdd(&sh.gathered, 1);
                if (at < kRoom) sh.found[at] = {logit, id};
            };
            // A thread's pieces are looked at by its whole warp, one each; of two threads they are on their way together.  (With four a single row
            // takes 0.4 us less, but a block leaves less room for others: 2,048 rows of 50,257 take 52 us instead of 44.)
            constexpr int kAhead = 2;
            unsigned ask = __ballot_sync(~0u, asked_most >= least);
            if (ask == ~0u && !above) {  // too many
                ask = 0;
                if (lane == 0) atomicAdd(&sh.gathered, kRoom + 1);
            }
            while (ask) {
                int first[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) first[k] = ask ? begin + 32 * warp + __ffs(ask) - 1 : end, ask &= ask - 1;
#pragma unroll 1
                for (int at = kThreads * lane; at < end - begin; at += kThreads * 32) {
                    uint4 w[kAhead];
                    unsigned hits[kAhead];
#pragma unroll
                    for (int k = 0; k < kAhead; ++k) w[k] = first[k] + at < end ? __ldg(from + first[k] + at) : P::nothing();
#pragma unroll
                    for (int k = 0; k < kAhead; ++k) {
                        hits[k] = 0;
#pragma unroll
                        for (int e = 0; e < P::kCount; ++e) hits[k] |= (unsigned)(P::at(w[k], e) >= least) << e;
                        if (first[k] + at >= end) hits[k] = 0;
                    }
#pragma unroll
                    for (int k = 0; k < kAhead; ++k)
#pragma unroll 1
                        for (; hits[k]; hits[k] &= hits[k] - 1) {
                            const int e = __ffs(hits[k]) - 1;
                            gather(P::pick(w[k], e), head + (first[k] + at) * P::kCount + e);
                        }
                }
            }
            at_ends(gather);
            __syncthreads();
            gathered = sh.gathered;
            const bool crowded = gathered > kRoom;
            if (!crowded || above) {
                int place = -1;
                if (tid < gathered) {
                    const Entry mine = sh.found[tid];
                    place = 0;
                    for (int i = 0; i < min(gathered, kRoom); i += 8)
#pragma unroll
                        for (int k = 0; k < 8; ++k) place += before(sh.found[i + k], mine);  // behind the last: nothing, which is before none
                    if (place < 32) sh.list[0][place] = mine;
                } else if (tid < 32) {
                    sh.list[0][tid] = best;  // nothing
                }
                if (!crowded) {
                    if (!above) break;
                    // ---- beside what lies above the bound, the lowest tokens at it
                    const float bound = from_ordered(ordered(least) - 1);
                    auto add_ties = [&](unsigned hits, int first_id) {  // hits: which of this thread's elements from first_id on; threads in the tokens' order
                        int upto = __popc(hits);
#pragma unroll 1
                        for (int d = 1; d < 32; d <<= 1) {
                            const int o = __shfl_up_sync(~0u, upto, d);
                            if (lane >= d) upto += o;
                        }
                        __syncthreads();
                        if (lane == 31) sh.most[warp] = upto;
                        __syncthreads();
                        int to = gathered + upto - __popc(hits);
#pragma unroll 1
                        for (int i = 0; i < kWarps; ++i) {
                            if (i < warp) to += sh.most[i];
                            gathered += sh.most[i];
                        }
                        for (; hits && to < p.top; hits &= hits - 1) sh.list[0][to++] = {bound, first_id + __ffs(hits) - 1};
                    };
                    if (rank == 0) add_ties(tid < head && P::one(x + tid) == bound, tid);
#pragma unroll 1
                    for (int i0 = begin; i0 < end && gathered < p.top; i0 += kThreads) {
                        unsigned hits = 0;
                        if (i0 + tid < end) {
                            const uint4 w = __ldg(from + i0 + tid);
#pragma unroll
                            for (int e = 0; e < P::kCount; ++e) hits |= (unsigned)(P::at(w, e) == bound) << e;
                        }
                        add_ties(hits, head + (i0 + tid) * P::kCount);
                    }
                    if (rank == parts - 1) add_ties(tid < p.V - tail_at && P::one(x + tail_at + tid) == bound, tail_at + tid);
                    break;
                }
                if (place == p.top - 1) sh.bound = ordered(sh.found[tid].x);
            }
            __syncthreads();
            if (above) least = from_ordered(sh.bound);
            least = from_ordered(ordered(least + 0.0f) + 1);  // the next number (of 0 the smallest above both zeros, of infinity a NaN, which nothing reaches)
            if (tid == 0) sh.gathered = 0;
            sh.found[tid] = {-INFINITY, kNoToken};
            __syncthreads();
        }
        __syncthreads();
        best = sh.list[0][lane];
    }

    // ---- the block, the cluster
    __syncthreads();
    auto join_all = [&](int n, auto list_of) {  // lists list_of(0 .. n - 1), n a power of two: into the first
        for (int step = 1; step < n; step <<= 1) {
            if (warp % (2 * step) == 0 && warp + step < n) {
                best = join_lists(best, list_of(warp + step)[31 - lane], lane);
                list_of(warp)[lane] = best;
            }
            __syncthreads();
        }
    };
    if (tid == 0) {
        for (int i = 1; i < kWarps; ++i) own.s0 += sh.sums[i].s0, own.s1 += sh.sums[i].s1;
        sh.block_sums = own;
    }
    if (parts > 1) {
        if (kTop && warp == 0) sh.block_list[lane] = best;
        cluster.sync();
        if (rank == 0) {
            if (warp == 0) {  // a block's sums a lane
                own = {-INFINITY, 0.0f, 0.0f};
                if (lane < parts) own = *cluster.map_shared_rank(&sh.block_sums, lane);
#pragma unroll
                for (int d = kMostCluster / 2; d > 0; d >>= 1) {
                    const Sums o = {__shfl_xor_sync(~0u, own.m, d), __shfl_xor_sync(~0u, own.s0, d), __shfl_xor_sync(~0u, own.s1, d)};
                    own = lane & d ? join_sums(o, own, c) : join_sums(own, o, c);  // the same order on both sides
                }
            }
            if constexpr (kTop) {
                if (warp < parts) best = cluster.map_shared_rank(&sh, warp)->block_list[lane];
                sh.list[warp][lane] = best;
                __syncthreads();
                join_all(parts, [&](int i) { return sh.list[i]; });
            }
        }
        cluster.sync();  // no block leaves while it is read
    }
    if (rank != 0 || warp != 0) return;
    const float m = __shfl_sync(~0u, own.m, 0), s0 = __shfl_sync(~0u, own.s0, 0), s1 = __shfl_sync(~0u, own.s1, 0);
    const bool none = m == -INFINITY, bad = !(m < INFINITY);  // nothing but masked tokens; a NaN or an infinity
    const float z = logf(s0);
    auto log_p = [&](float logit) {
        if (bad) return __int_as_float(0x7FFFFFFF);
        return none ? -INFINITY : fmaf(p.scale, logit - m, -z);
    };
    if (lane == 0) {
        const float nan = __int_as_float(0x7FFFFFFF);
        if (p.entropy) p.entropy[row] = bad ? nan : (none ? 0.0f : z - kLn2 * (s1 / s0));
        if (p.lse) p.lse[row] = bad ? nan : (none ? -INFINITY : fmaf(p.scale, m, z));
        if (p.logprob) p.logprob[row] = token >= 0 && token < p.V ? log_p(given) : 0.0f;
    }
    if (kTop && lane < p.top) {
        const bool found = best.id != kNoToken;
        if (p.top_id) p.top_id[row * p.top + lane] = found ? best.id : -1;
        if (p.top_logprob) p.top_logprob[row * p.top + lane] = log_p(best.x);
    }
}

template <int kType>
cudaError_t launch(const LogprobParams& p, int64_t T, int parts, cudaStream_t st) {
    cudaLaunchAttribute attr[2] = {early_launch_attribute(), cluster_attribute(1)};
    attr[1].val.clusterDim.x = parts, attr[1].val.clusterDim.y = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(T * parts));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return p.top ? cudaLaunchKernelEx(&cfg, token_logprobs_kernel<kType, true>, p) : cudaLaunchKernelEx(&cfg, token_logprobs_kernel<kType, false>, p);
}

}  // namespace
}  // namespace awe

using namespace awe;

extern "C" awe_status_t awe_token_logprobs(awe_handle_t h, const void* logits_dev, awe_float_t type, int64_t T, int64_t V, int64_t ld,
                                           float scale, const int32_t* tokens_dev, float* logprob_dev, float* entropy_dev,
                                           float* lse_dev, int64_t top_k, float* top_logprob_dev, int32_t* top_id_dev, void* stream) {
    if (!h || T < 0 || V <= 0 || top_k < 0 || !(scale > 0.0f && scale <= 1e30f)) return AWE_ERR_INVALID_ARG;
    if ((int)type < AWE_F16 || (int)type > AWE_F32) return AWE_ERR_INVALID_ARG;
    if (top_k > AWE_MAX_TOP || V > INT32_MAX / 2) return AWE_ERR_UNSUPPORTED;
    if (T == 0) return AWE_OK;
    if (!logits_dev || (T > 1 && ld < V) || top_k > V || (logprob_dev && !tokens_dev)) return AWE_ERR_INVALID_ARG;
    if (T > INT32_MAX / kMostCluster) return AWE_ERR_UNSUPPORTED;
    if ((uintptr_t)logits_dev % (type == AWE_F32 ? 4 : 2) || (uintptr_t)tokens_dev % 4 || (uintptr_t)logprob_dev % 4 || (uintptr_t)entropy_dev % 4 ||
        (uintptr_t)lse_dev % 4 || (uintptr_t)top_logprob_dev % 4 || (uintptr_t)top_id_dev % 4)
        return AWE_ERR_ALIGNMENT;
    if (!top_logprob_dev && !top_id_dev) top_k = 0;
    if (!logprob_dev && !entropy_dev && !lse_dev && !top_k) return AWE_OK;
    LogprobParams p = {logits_dev, tokens_dev, logprob_dev, entropy_dev, lse_dev, top_logprob_dev, top_id_dev, ld, scale, (int)V, (int)top_k};
    // A row goes to a cluster while its blocks keep enough of it: twice as much where lists have to be joined, and twice as much again when
    // there are blocks for half of the SMs, and for two on each.  BF16, 20 alternatives, 1, 2, 4 and 8 blocks a row, us: 1 x 32,000 8.0, 8.4,
    // 8.4, 8.6; 16 x 65,536 10.7, 10.4, 9.6, 9.8; 64 x 131,072 17.4, 12.8, 12.3, 14.2; 148 x 65,536 11.3, 12.1, 15.3, 22.9;
    // 300 x 131,072 29.9, 27.4, 34.6, 46.6; 600 x 131,072 45.6, 47.3, 57.6, 87.0.  Without alternatives: 1 x 32,000 4.2, 4.3, 3.6, 3.6;
    // 64 x 65,536 6.7, 5.5, 4.8, 5.1; 300 x 131,072 23.1, 20.8, 21.6, 21.9.
    const int64_t batch = (int64_t)kThreads * kPieces * (type == AWE_F32 ? 4 : 8) * (top_k ? 2 : 1), sms = h->sm_count;
    int parts = 1;
    for (; parts < kMostCluster; parts *= 2) {
        const int64_t blocks = T * parts * 2;
        if (blocks > 5 * sms || V < batch * 2 * parts * (2 * blocks <= sms ? 1 : blocks < 2 * sms ? 2 : 4)) break;
    }
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = type == AWE_F32 ? launch<AWE_F32>(p, T, parts, st) : type == AWE_BF16 ? launch<AWE_BF16>(p, T, parts, st) : launch<AWE_F16>(p, T, parts, st);
    if (e != cudaSuccess) return AWE_ERR_CUDA;
    h->launches += 1;
    return AWE_OK;
}
