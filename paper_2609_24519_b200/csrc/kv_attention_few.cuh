// What the kernels for few query rows share, over the cache of 8 bits (awe_kv_attention.cu) and of 4 (awe_kv4_attention.cu): how the
// steps are dealt out, which tokens rows see, how the warps of a block are joined.
#pragma once
#include <algorithm>

#include "kv_attention.cuh"

namespace awe {
namespace attn_few {

using namespace serve;

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kWholeTokens = 256;
constexpr int64_t kWholeScans = 1 << 19;

// The steps of one request: tokens [lo, hi) in steps of kStepTokens (a tile for each warp), for each of `units` units.
struct Request {
    int q0, n, ctx, lo, steps, units;
};
template <int kRows, int kStepTokens>
__device__ __forceinline__ Request request_of(const AttnParams& p, int b) {
    Request r;
    r.q0 = min(max(p.q_start[b], 0), (int)p.T);
    r.n = max(min(p.q_start[b + 1], (int)p.T) - r.q0, 0);
    // no token beyond the table's row
    r.ctx = (int)min((int64_t)max(p.ctx_len[b], 0), (int64_t)p.max_pages << p.page_log2);
    const int64_t first = (int64_t)p.ctx_len[b] - r.n + 1 - p.window;  // first token that any of its queries sees
    r.lo = p.window > 0 && first > 0 ? (int)min(first, (int64_t)r.ctx) & ~(kStepTokens - 1) : 0;
    r.steps = max((int)(((unsigned)(r.ctx - r.lo) + kStepTokens - 1) / kStepTokens), 1);  // one at least: its rows are to be written
    r.units = (r.n * p.group + kRows - 1) / kRows * p.heads;
    return r;
}

// Which steps are block `number`'s, by an exclusive sum of units x steps over the requests: [begin, end), the request that `begin` lies in
// and where its steps start.  False if there are none.
struct Search {
    int64_t scan[kWarps];
    int found_b;
    int64_t found_at;
};
struct Mine {
    int64_t begin, end, at;
    int b;
};
template <int kRows, int kStepTokens>
__device__ __forceinline__ bool find_steps(const AttnParams& p, Search& sh, Mine& mine_out, int number) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int64_t total = 0;
    for (int pass = 0; pass < 2; ++pass) {
        const int64_t mine = pass ? Deal(total, p.blocks).begin(number) : 0;
        int64_t sum = 0;
        for (int b0 = 0; b0 < p.B; b0 += kThreads) {
            const int b = b0 + tid;
            int64_t w = 0;
            if (b < p.B) {
                const Request r = request_of<kRows, kStepTokens>(p, b);
                w = p.whole ? r.units : (int64_t)r.units * r.steps;
            }
            int64_t inc = w;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int64_t o = __shfl_up_sync(~0u, inc, d);
                if (lane >= d) inc += o;
            }
            __syncthreads();
            if (lane == 31) sh.scan[warp] = inc;
            __syncthreads();
            int64_t before = sum;
#pragma unroll
            for (int i = 0; i < kWarps; ++i) {
                if (i < warp) before += sh.scan[i];
                sum += sh.scan[i];
            }
            const int64_t at = before + inc - w;
            if (pass && b < p.B) {
                if (blockIdx.x == 0) p.unit_steps[b] = at;
                if (at <= mine && mine < at + w) {
                    sh.found_b = b;
                    sh.found_at = at;
                }
            }
        }
        total = sum;
    }
    if (blockIdx.x == 0 && tid == 0) p.unit_steps[p.B] = total;
    __syncthreads();
    const Deal deal(total, p.blocks);
    if (number >= deal.blocks || total == 0) return false;
    mine_out = {deal.begin(number), deal.begin(number + 1), sh.found_at, sh.found_b};
    return true;
}

// A query row's 32-bit words in FP16: BF16 ones, and if kScaled all, are scaled by a power of two (query_exponent), which `factor` takes
// back.  The row lies in the four threads of a lane group.
template <bool kBf16, bool kScaled, int kWords>
__device__ __forceinline__ void query_to_fp16(uint32_t (&raw)[kWords][2], float& factor) {
    if constexpr (kBf16 || kScaled) {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < kWords; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float2 f = Half<kBf16>::unpack(raw[i][j]);
                m = fmaxf(m, fmaxf(fabsf(f.x), fabsf(f.y)));
            }
        m = fmaxf(m, __shfl_xor_sync(~0u, m, 1));
        m = fmaxf(m, __shfl_xor_sync(~0u, m, 2));
        const int e = query_exponent((int)(__float_as_uint(m) >> 23));
        const float down = power_of_2(15 - e);
        factor *= power_of_2(e - 15);
#pragma unroll
        for (int i = 0; i < kWords; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float2 f = Half<kBf16>::unpack(raw[i][j]);
                raw[i][j] = Half<false>::pack(f.x * down, f.y * down);
            }
    }
}
// Tokens [lo, hi) that query `query` of request b sees; none where it is not live.
__device__ __forceinline__ void visible(const AttnParams& p, const Request& r, int b, int query, bool live, int& lo, int& hi) {
    const int64_t place = (int64_t)p.ctx_len[b] - r.n + query;  // of the query among its request's tokens
    hi = p.causal ? (int)min((int64_t)r.ctx, place + 1) : r.ctx;
    lo = p.window > 0 && place + 1 > p.window ? (int)min(place + 1 - p.window, (int64_t)r.ctx) : 0;
    if (!live || hi < 0) hi = 0;
}

// Tokens [all_lo, all_hi) that every row of a unit sees, and [any_lo, any_hi) that some row sees: the pages of others are not
// followed, which a window may have given up.
struct Sees {
    int all_lo, all_hi, any_lo, any_hi;
};
template <int kNT>
__device__ __forceinline__ Sees sees_of(const int (&see_lo)[kNT][2], const int (&see_hi)[kNT][2], int n_rows, int t) {
    int all_lo = 0, all_hi = 0x7FFFFFFF;
#pragma unroll
    for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (8 * nt + 2 * t + j < n_rows) all_lo = max(all_lo, see_lo[nt][j]), all_hi = min(all_hi, see_hi[nt][j]);
    all_lo = __reduce_max_sync(~0u, all_lo);
    all_hi = __reduce_min_sync(~0u, all_hi);
    int any_lo = 0x7FFFFFFF, any_hi = 0;
#pragma unroll
    for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (see_lo[nt][j] < see_hi[nt][j]) any_lo = min(any_lo, see_lo[nt][j]), any_hi = max(any_hi, see_hi[nt][j]);
    any_lo = __reduce_min_sync(~0u, any_lo);
    any_hi = __reduce_max_sync(~0u, any_hi);
    return {all_lo, all_hi, any_lo, any_hi};
}

// ln(2^m sum) for a whole m.
__device__ __forceinline__ float log_sum(float m, float sum) {
    int e;
    const float f = frexpf(sum, &e);
    return (m + (float)e + log2f(f)) * 0.69314718056f;
}

// The result of a unit, or its part, from the warps' vectors and (reference, sum of the weights, sum for the logarithm).
// kWholeRef: references are whole numbers.
template <int kD, int kRows, bool kBf16, bool kWholeRef = false>
__device__ __forceinline__ void finish_unit(const AttnParams& p, const Request& r, const float* join_vec, const float4* join_stat, int step0, int step1,
                                            int head, int row0, int n_rows) {
    using T16 = typename Half<kBf16>::type;
    constexpr int kVecPitch = kD + 4;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool whole = step0 == 0 && step1 == r.steps;
    const int slot = 2 * blockIdx.x + (step0 == 0);
    for (int row = warp; row < n_rows; row += kWarps) {
        float4 st[kWarps];
        float m = -INFINITY, total_sum = 0.0f, total_lse = 0.0f, a[kWarps];
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            st[w] = join_stat[w * kRows + row];
            m = fmaxf(m, st[w].x);
        }
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            a[w] = st[w].x == -INFINITY ? (st[w].y == 0.0f ? 0.0f : 1.0f) : exp2_approx(st[w].x - m);
            total_sum = fmaf(st[w].y, a[w], total_sum);
            total_lse = fmaf(st[w].z, a[w], total_lse);
        }
        const int query = (row0 + row) / p.group, qh = head * p.group + (row0 + row) % p.group;
        const int64_t token = r.q0 + query;
        const float inv = total_sum == 0.0f ? 0.0f : 1.0f / total_sum;
        T16* dst = reinterpret_cast<T16*>(p.out) + token * p.ldo + (int64_t)qh * kD;
        for (int d = 4 * lane; d < kD; d += 128) {
            float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float4 y = *reinterpret_cast<const float4*>(join_vec + (w * kRows + row) * kVecPitch + d);
                x.x = fmaf(y.x, a[w], x.x), x.y = fmaf(y.y, a[w], x.y), x.z = fmaf(y.z, a[w], x.z), x.w = fmaf(y.w, a[w], x.w);
            }
            if (whole)
                *reinterpret_cast<uint2*>(dst + d) =
                    make_uint2(Half<kBf16>::pack(x.x * inv, x.y * inv), Half<kBf16>::pack(x.z * inv, x.w * inv));
            else
                *reinterpret_cast<float4*>(p.part_vec + ((int64_t)slot * kRows + row) * kD + d) = x;
        }
        if (lane == 0) {
            if (!whole) p.part_stat[(int64_t)slot * kRows + row] = make_float4(m, total_sum, total_lse, 0.0f);
            else if (p.lse)
                p.lse[token * p.heads * p.group + qh] = total_lse == 0.0f ? -INFINITY : kWholeRef ? log_sum(m, total_lse) : (m + log2f(total_lse)) * 0.69314718056f;
        }
    }
}

// Query rows a unit holds: 16 where a request has more than 8 on average (their cache bytes are then read once),
// else 8; head dimension 256 leaves no registers for 16.
inline int row_tiles(int64_t T, int64_t B, int64_t group, int64_t head_dim) {
    return head_dim < 256 && T * group > 8 * B ? 2 : 1;
}

struct Workspace {
    size_t vec, stat, total;
};
inline Workspace workspace_of(int blocks, int rows, int64_t head_dim, int64_t B) {
    Workspace w;
    w.vec = (size_t)round_up((B + 1) * 8, 256);
    w.stat = w.vec + (size_t)2 * blocks * rows * head_dim * 4;
    w.total = w.stat + (size_t)2 * blocks * rows * 16;
    return w;
}

// Blocks of the launch and their places in the workspace.  Short contexts: a block per unit and no second launch.  Each block scans
// all requests, so it pays while the units times the requests are few: up to 256 tokens for one query, 8 heads of 4 queries each, us
// whole / in parts with the join (8 bits): 1 request 7.0 / 7.6, 64 16.2 / 17.6, 128 25.2 / 26.6, 256 50 / 47, 2,048 902 / 337; 1 head of
// 8: 128 7.6 / 11.1, 512 20.7 / 22.3, 1,024 47 / 38.
inline void place_few(AttnParams& p, int step_tokens, int blocks, int nt, int64_t head_dim, int64_t tokens, void* workspace_dev) {
    if (p.window > 0) tokens = std::min(tokens, p.window + p.T / p.B + step_tokens);
    const int64_t units = (p.T * p.group / (8 * nt) + p.B) * p.heads;
    p.whole = tokens <= kWholeTokens && units * p.B <= kWholeScans;
    const Workspace w = workspace_of(blocks, 8 * nt, head_dim, p.B);
    p.unit_steps = (int64_t*)workspace_dev;
    p.part_vec = (float*)((uint8_t*)workspace_dev + w.vec);
    p.part_stat = (float4*)((uint8_t*)workspace_dev + w.stat);
    p.blocks = p.whole ? (int)units : blocks;
}

}  // namespace attn_few
}  // namespace awe
