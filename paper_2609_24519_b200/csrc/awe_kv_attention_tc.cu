// Attention over the paged cache of 8 or of 4 bits for prompts, on tcgen05.  The formulas are those of awe_kv_attention.cu and
// awe_kv4_attention.cu.
//
// A unit of work is (request, cache head, 256 query rows), two tiles of 128 rows that share every key and value.  Per step
// of 128 tokens four warps unpack the keys and values to FP16 (exact) in shared memory, one thread issues
//   S = Q K^T   (Q and K from shared memory, S in tensor memory)   and   O += P V   (P from tensor memory, V from shared),
// and four warps per tile turn S into P, a thread per query row.  The two tiles take turns on the tensor cores, so that one's
// softmax runs beside the other's products.
//
// Scales.  The keys' scale of 16 tokens of a page multiplies the scores in FP32.  The values' scale vs is folded into P as
// an addition to the exponent: P = exp2(s + log2 vs - m) with m 10 to 15 below the largest s + log2 vs seen so far, so
// that P rounds to FP16 as well as it can for what it contributes, whatever the scales; the divisor is the sum of
// 2^-12 P / vs in FP32 (the power of two keeps it in range for every scale that the cache write stores, 2^-107 to 2^121).
// m moves only when a score passes it by more than 15, which rescales O in tensor memory; that is rare after the first step.
// Tokens whose page has value scale 0 stand for zeros whatever their bytes, and weigh in the divisor alone: their P is 0, so that
// they neither add to O nor move m, and their exponentials are summed apart, against a maximum of their own, in a pass that only
// steps with such pages take; the two sums meet at the end.
//
// The cache of 4 bits has a scale for every token.  Its values, scale times (code - zero), are exact in FP16, so they are unpacked whole
// and the softmax knows no scales: P is the weight alone, rounded by 2^-11 of itself or 2^-34 of the largest weight (m, which moves by whole
// numbers, stays 9 to 15 below the largest s), whatever the values' scales.  A word's eight codes come apart in the order 0 4 1 5 2 6 3 7, in which the operands keep them: queries are
// brought into it, results back.  2,048 queries of 8,192 tokens, 32 / 8 heads of 128: 347 us, 690 TFLOP/s; with S read twice, as for 8 bits, 373.
//
// All steps of all units in a row are dealt out evenly to one block per SM; units that were cut are joined by a second
// kernel in the order of the tokens.  A small kernel before lists the units' steps, which causality makes uneven.
#include <algorithm>
#include <type_traits>

#include "gemm_common.cuh"
#include "kv4.cuh"
#include "kv_attention.cuh"
#include "ptx_serve.cuh"

namespace awe {
namespace {

using namespace serve;

constexpr int kRows = 256;      // query rows of a unit
constexpr int kStep = 128;      // tokens of a step
constexpr int kSoftWarps = 8, kUnpackWarps = 4, kMultiplier = kSoftWarps + kUnpackWarps, kThreads = 32 * (kMultiplier + 1);
constexpr int kTmemCols = 512;
constexpr int kPlanThreads = 1024;

struct TcAttnParams {
    AttnParams a;
    int64_t* tile_steps;   // [tiles + 1]: exclusive sum over the row tiles of heads x steps
    int2* tile_of;         // [tiles]: request, row tile
    int32_t* tile_base;    // [B + 1]: first row tile of each request
    int max_tiles;         // what T queries of B requests can have; starts that ask for more get no more
    unsigned int* status;
};

struct Unit {
    int b, q0, n, ctx, row0, rows, lo, steps;
    int first, end;  // tokens that some row may see: the pages of others are not followed, which a window may have given up
    int64_t place0;  // of the request's first query among its tokens
};
__device__ __forceinline__ Unit unit_of(const AttnParams& p, int b, int tile) {
    Unit u;
    u.b = b;
    u.q0 = min(max(p.q_start[b], 0), (int)p.T);
    u.n = max(min(p.q_start[b + 1], (int)p.T) - u.q0, 0);
    u.ctx = (int)min((int64_t)max(p.ctx_len[b], 0), (int64_t)p.max_pages << p.page_log2);  // no token beyond the table's row
    u.place0 = (int64_t)p.ctx_len[b] - u.n;
    u.row0 = tile * kRows;
    u.rows = min(kRows, u.n * p.group - u.row0);
    const int64_t first = u.place0 + u.row0 / p.group, last = u.place0 + (u.row0 + u.rows - 1) / p.group;
    const int64_t hi = p.causal ? min((int64_t)u.ctx, last + 1) : (int64_t)u.ctx;
    u.first = p.window > 0 && first + 1 > p.window ? (int)min(first + 1 - p.window, (int64_t)u.ctx) : 0;
    u.lo = u.first & ~(kStep - 1);
    u.end = (int)max(hi, (int64_t)0);
    u.steps = max((int)((hi - u.lo + kStep - 1) / kStep), 1);  // one at least: its rows are to be written
    return u;
}
__device__ __forceinline__ int tiles_of(const AttnParams& p, int b) {
    const int q0 = min(max(p.q_start[b], 0), (int)p.T), n = max(min(p.q_start[b + 1], (int)p.T) - q0, 0);
    return (n * p.group + kRows - 1) / kRows;
}

// Exclusive sum over a block of kPlanThreads threads.
__device__ __forceinline__ int64_t block_scan(int64_t x, int64_t* warp_sums, int64_t* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t inc = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t o = __shfl_up_sync(~0u, inc, d);
        if (lane >= d) inc += o;
    }
    __syncthreads();
    if (lane == 31) warp_sums[warp] = inc;
    __syncthreads();
    int64_t before = 0, all = 0;
    for (int w = 0; w < kPlanThreads / 32; ++w) {
        if (w < warp) before += warp_sums[w];
        all += warp_sums[w];
    }
    *total = all;
    return before + inc - x;
}

__global__ void __launch_bounds__(kPlanThreads) kv_attention_units_kernel(const TcAttnParams p) {
    __shared__ int64_t warp_sums[kPlanThreads / 32];
    grid_wait();
    int64_t base = 0, all;
    for (int b0 = 0; b0 < p.a.B; b0 += kPlanThreads) {
        const int b = b0 + threadIdx.x, n = b < p.a.B ? tiles_of(p.a, b) : 0;
        const int64_t at = base + block_scan(n, warp_sums, &all);
        if (b < p.a.B) p.tile_base[b] = (int)at;
        base += all;
    }
    const int tiles = (int)min(base, (int64_t)p.max_tiles);
    if (threadIdx.x == 0) p.tile_base[p.a.B] = tiles;
    __syncthreads();
    int64_t sum = 0;
    for (int t0 = 0; t0 < tiles; t0 += kPlanThreads) {
        const int t = t0 + threadIdx.x;
        int64_t w = 0;
        if (t < tiles) {
            int b = 0;  // last request whose first tile is not behind t
            for (int n = p.a.B; n > 1;) {
                const int half = n >> 1;
                if (p.tile_base[b + half] <= t) b += half;
                n -= half;
            }
            const int tile = t - p.tile_base[b];
            p.tile_of[t] = make_int2(b, tile);
            w = (int64_t)unit_of(p.a, b, tile).steps * p.a.heads;
        }
        const int64_t at = sum + block_scan(w, warp_sums, &all);
        if (t < tiles) p.tile_steps[t] = at;
        sum += all;
    }
    if (threadIdx.x == 0) p.tile_steps[tiles] = sum;
}

constexpr int kSharedBytes = 3 * 1024;  // room for Shared
constexpr int kFewTokens = 32;  // of more, errors are at most 1.4 times those of weights in FP32, here 1.3; 2,048 FP16 queries of 8,192 tokens 341 -> 347 us
constexpr float kDivisorUnit = 1.0f / 4096, kDivisorLog2 = 12.0f;

template <int kD>
struct Config {
    static constexpr int kQBytes = 128 * kD * 2, kKBytes = kStep * kD * 2;  // of one tile
    static constexpr int kQAt = 0, kKAt = 2 * kQBytes, kVAt = kKAt + 2 * kKBytes, kEnd = kVAt + 2 * kKBytes;
    // 195 KB for dimension 128, and no more: with the 1 KB that every block has besides, 196 KB of the SM's 256 are shared memory
    // and the rest caches the loads; the next larger split costs 12 us of 374 (2,048 queries of 8,192 tokens).
    static constexpr int kNeeded = kEnd + kSharedBytes;
    static_assert(kD != 128 || kNeeded <= 195 * 1024, "split of the SM's memory");
    // A block takes all of tensor memory, so a second one must not fit beside it.
    static constexpr int kSmemBytes = kNeeded > 120 * 1024 ? kNeeded : 120 * 1024;
};

struct Shared {
    uint64_t q_full[2], k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_full[2], o_done[2];
    uint64_t c_full[4];  // constants of a step: four of them, so that no softmax warp can fall a round behind
    uint32_t tmem_base;
    volatile uint32_t abort_flag;
    float4 constants[4][kStep / 16];  // of 16 tokens: key scale, log2 of the value scale, kDivisorUnit over it
    uint32_t unvalued[4];             // of a step: which 16 tokens have value scale 0; 4 bits: which have no page
    float2 unvalued_sum[kRows];       // of a query row over those: reference, sum of the exponentials
};
static_assert(sizeof(Shared) <= kSharedBytes, "shared memory behind the tiles");

// Descriptor of an operand whose rows run along the contraction: 64 columns (128 bytes) per row, 128-byte swizzle, 8-row
// groups 1024 bytes apart, blocks of 64 columns `block_bytes` apart.
__device__ __forceinline__ uint64_t smem_desc_mn_sw128(uint32_t addr, uint32_t block_bytes) {
    uint64_t d = 0;
    d |= (uint64_t)((addr & 0x3FFFF) >> 4);
    d |= (uint64_t)(block_bytes >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

__device__ __noinline__ bool wait_long(volatile uint32_t* abort_flag, uint32_t bar, uint32_t parity, unsigned int* status, int site) {
    return gemm::bounded_wait_ns(abort_flag, bar, parity, status, site, gemm::kWaitLimitNs);
}

// The factor of 16 tokens' scores.  It is not negative, and not 0, so that a hidden score stays -inf under it.
__device__ __forceinline__ float factor_of(float key_scale, float cq) { return fmaxf(key_scale * cq, 1.17549435e-38f); }

// Adds the exponentials of a step's tokens whose page has value scale 0 (`groups`: which 16 of them) to a query row's sum of
// those; the row's scores lie in tensor memory at `scores`, it sees the step's tokens [lo, hi).
__device__ __forceinline__ void add_unvalued(Shared* sh, uint32_t groups, int slot, uint32_t scores, int row, int lo, int hi, float cq) {
    float2 own = sh->unvalued_sum[row];
#pragma unroll 1
    for (int g = 0; g < kStep / 16; ++g, lo -= 16, hi -= 16) {
        if (!(groups >> g & 1)) continue;
        uint32_t v[16];
        ptx::tmem_ld_32x16(scores + 16 * g, v);
        ptx::tmem_wait_ld();
        if (lo < min(hi, 16) && hi > 0) {  // this row sees some of them
            const float a = factor_of(sh->constants[slot][g].x, cq);
            float m = -INFINITY;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                if (e < lo || e >= hi) v[e] = 0xFF800000u;
                m = fmaxf(m, __uint_as_float(v[e]));
            }
            m = fmaxf(own.x, m * a);
            own.y *= exp2_approx(own.x - m);
#pragma unroll
            for (int e = 0; e < 16; ++e) own.y += exp2_approx(fmaf(__uint_as_float(v[e]), a, -m));
            own.x = m;
        }
        __syncwarp();
    }
    sh->unvalued_sum[row] = own;
}

template <int kD, bool kBf16, bool kFour>
__global__ void __launch_bounds__(kThreads, 1) kv_attention_tc_kernel(const TcAttnParams tp) {
    using C = Config<kD>;
    using T16 = typename Half<kBf16>::type;
    // FP16 outputs over the cache of 4 bits: where a warp has a row that sees few tokens, the divisor is the sum of the rounded weights, so that the
    // rounding of a token that dominates cancels and a row of one token has exactly its values.  (BF16 outputs round eight times as much themselves.)
    constexpr bool kRounded = kFour && !kBf16;
    const AttnParams& p = tp.a;
    extern __shared__ __align__(1024) uint8_t smem[];  // swizzled tiles
    const uint32_t base = ptx::smem_u32(smem);
    Shared* sh = reinterpret_cast<Shared*>(smem + C::kEnd);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            ptx::mbar_init(ptx::smem_u32(&sh->q_full[i]), 4);
            ptx::mbar_init(ptx::smem_u32(&sh->k_full[i]), kUnpackWarps);
            ptx::mbar_init(ptx::smem_u32(&sh->v_full[i]), kUnpackWarps);
            ptx::mbar_init(ptx::smem_u32(&sh->p_full[i]), 4);
            ptx::mbar_init(ptx::smem_u32(&sh->k_empty[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&sh->v_empty[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&sh->s_full[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&sh->o_done[i]), 1);
        }
        for (int i = 0; i < 4; ++i) ptx::mbar_init(ptx::smem_u32(&sh->c_full[i]), 1);
        sh->abort_flag = 0;
        ptx::fence_mbar_init();
    }
    if (warp == kMultiplier) {
        ptx::tmem_alloc(ptx::smem_u32(&sh->tmem_base), kTmemCols);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    grid_wait();
    const uint32_t tmem = sh->tmem_base;
    const uint32_t s_at[2] = {tmem, tmem + 128}, o_at[2] = {tmem + 256, tmem + 256 + kD};  // P takes the first 64 columns of S
    auto wait = [&](uint64_t& bar, uint32_t parity, int site) {
        const uint32_t at = ptx::smem_u32(&bar);
        return ptx::mbar_try_wait(at, parity) || wait_long(&sh->abort_flag, at, parity, tp.status, site);
    };

    // ---- my steps
    const int tiles = tp.tile_base[p.B];
    const int64_t total = tp.tile_steps[tiles];
    const Deal deal(total, p.blocks);
    const bool mine = (int)blockIdx.x < deal.blocks && total > 0;
    const int64_t begin = mine ? deal.begin(blockIdx.x) : 0, end = mine ? deal.begin(blockIdx.x + 1) : 0;
    int tile = 0;  // last row tile that begins at or before `begin`
    for (int n = tiles; n > 1;) {
        const int half = n >> 1;
        if (tp.tile_steps[tile + half] <= begin) tile += half;
        n -= half;
    }
    // Calls f(unit, head, first step, end step, whether that is the whole unit) for each part of a unit; f says whether to go on.
    auto for_parts = [&](auto f) {
        int t = tile;
        for (int64_t pos = begin; pos < end;) {
            while (pos >= tp.tile_steps[t + 1]) ++t;
            const int2 id = tp.tile_of[t];
            const Unit u = unit_of(p, id.x, id.y);
            const int64_t in = pos - tp.tile_steps[t];
            const int head = (int)(in / u.steps), s0 = (int)(in % u.steps), s1 = (int)min((int64_t)u.steps, s0 + end - pos);
            if (!f(u, head, s0, s1)) return;
            pos += s1 - s0;
        }
    };

    if (warp == kMultiplier) {
        if (lane == 0) {
            constexpr uint32_t kIdescS = (1u << 4) | ((uint32_t)(kStep >> 3) << 17) | (8u << 24);
            constexpr uint32_t kIdescO = (1u << 4) | (1u << 16) | ((uint32_t)(kD >> 3) << 17) | (8u << 24);
            uint32_t step = 0, step_of[2] = {0, 0}, part_of[2] = {0, 0};  // steps and parts so far, in all and of each tile
            for_parts([&](const Unit& u, int, int s0, int s1) {
                const int n_tiles = u.rows > 128 ? 2 : 1, n = s1 - s0;
                auto scores = [&](int t, uint32_t at_step, bool last) {  // S = Q K^T of tile t
                    const uint64_t q = ptx::smem_desc_k_sw128(base + C::kQAt + t * C::kQBytes);
                    const uint64_t k = ptx::smem_desc_k_sw128(base + C::kKAt + (at_step & 1) * C::kKBytes);
#pragma unroll
                    for (int c = 0; c < kD / 16; ++c)
                        ptx::mma_f16(s_at[t], q + ((c >> 2) * 128 * 128 + (c & 3) * 32) / 16, k + ((c >> 2) * kStep * 128 + (c & 3) * 32) / 16, kIdescS, c != 0);
                    ptx::mma_commit(ptx::smem_u32(&sh->s_full[t]));
                    if (last) ptx::mma_commit(ptx::smem_u32(&sh->k_empty[at_step & 1]));
                };
                if (!wait(sh->k_full[step & 1], (step >> 1) & 1, 30)) return false;
                for (int t = 0; t < n_tiles; ++t) {
                    if (!wait(sh->q_full[t], part_of[t] & 1, 31)) return false;
                    ++part_of[t];
                    ptx::tc_fence_after();
                    scores(t, step, t == n_tiles - 1);
                }
                for (int j = 0; j < n; ++j, ++step) {
                    if (!wait(sh->v_full[step & 1], (step >> 1) & 1, 32)) return false;
                    for (int t = 0; t < n_tiles; ++t) {
                        if (!wait(sh->p_full[t], step_of[t] & 1, 33)) return false;
                        ++step_of[t];
                        ptx::tc_fence_after();
                        const uint64_t v = smem_desc_mn_sw128(base + C::kVAt + (step & 1) * C::kKBytes, kStep * 128);
#pragma unroll
                        for (int c = 0; c < kStep / 16; ++c)
                            ptx::mma_f16_ta(o_at[t], s_at[t] + c * 8, v + c * (16 * 128 / 16), kIdescO, j > 0 || c != 0);
                        ptx::mma_commit(ptx::smem_u32(&sh->o_done[t]));
                        if (t == n_tiles - 1) ptx::mma_commit(ptx::smem_u32(&sh->v_empty[step & 1]));
                        if (j + 1 < n) {
                            if (t == 0 && !wait(sh->k_full[(step + 1) & 1], ((step + 1) >> 1) & 1, 30)) return false;
                            ptx::tc_fence_after();
                            scores(t, step + 1, t == n_tiles - 1);
                        }
                    }
                }
                return true;
            });
        }
    } else if (kFour && warp >= kSoftWarps) {  // ---- unpack keys and values of 4 bits
        constexpr int kPieces = kD / 32;  // 16-byte pieces per token
        constexpr int kPassRows = 32 * kUnpackWarps / kPieces, kPasses = kStep / kPassRows;  // tokens per pass
        const int thread = tid - 32 * kSoftWarps, c = thread % kPieces, r = thread / kPieces;
        uint32_t step = 0;
        for_parts([&](const Unit& u, int head, int s0, int s1) {
            const int32_t* table = p.table + (int64_t)u.b * p.ld_table;
            auto page_of = [&](int j) {  // lanes below 8: page of their 16 tokens of step j, -1 where there is none
                const int tok = u.lo + j * kStep + 16 * lane;
                int page = -1;
                if (j < s1 && lane < kStep / 16 && tok < u.end && tok + 16 > u.first) {
                    page = table[tok >> p.page_log2];
                    if (page < 0 || page >= p.n_pages) page = -1;
                }
                return page;
            };
            uint4 kr[kPasses], vr[kPasses];
            uint32_t kw[kPasses], vw[kPasses];  // parameter words
            uint32_t at[kPasses];               // rows of the pieces of a step; ~0 where there is nothing
            auto places = [&](int pages, int j) {
                const int place = (u.lo + j * kStep) & ((1 << p.page_log2) - 1);
#pragma unroll
                for (int i = 0; i < kPasses; ++i) {
                    const int row = i * kPassRows + r, page = __shfl_sync(~0u, pages, row >> 4);
                    const uint32_t block = (uint32_t)(page * p.heads + head) << p.page_log2;
                    at[i] = page < 0 ? ~0u : block + ((place + row) & ((1 << p.page_log2) - 1));
                }
            };
            auto load = [&](const int8_t* pool, const uint16_t* params, uint4 (&x)[kPasses], uint32_t (&words)[kPasses]) {
#pragma unroll
                for (int i = 0; i < kPasses; ++i) {
                    x[i] = make_uint4(0, 0, 0, 0), words[i] = 0;  // become zeros, under a weight of 0
                    if (at[i] != ~0u) {
                        x[i] = __ldg(reinterpret_cast<const uint4*>(pool) + ((uint64_t)at[i] * kPieces + c));
                        words[i] = __ldg(params + at[i]);
                    }
                }
            };
            auto store = [&](uint32_t to, uint4 (&x)[kPasses], const uint32_t (&words)[kPasses]) {
                const int swap = kPieces == 4 ? c >> 1 : 0;  // the two blocks' threads write opposite halves first: no bank twice
#pragma unroll
                for (int i = 0; i < kPasses; ++i) {
                    const int row = i * kPassRows + r;
                    if (swap) x[i] = make_uint4(x[i].z, x[i].w, x[i].x, x[i].y);
                    const __half2 scale = __float2half2_rn(kv4_scale(words[i]));
                    const Kv4Zeros zero(__byte_perm(words[i], 0, 0x1010));
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t x0 = (&x[i].x)[w], x1 = x0 >> 8;
                        const uint32_t h0 = mul2(kv4_low_codes(x0, zero), scale), h1 = mul2(kv4_high_codes(x0, zero), scale);
                        const uint32_t h2 = mul2(kv4_low_codes(x1, zero), scale), h3 = mul2(kv4_high_codes(x1, zero), scale);
                        const uint32_t at = to + (c >> 1) * kStep * 128 + row * 128 + ((((4 * c + (w ^ (2 * swap))) & 7) ^ (row & 7)) << 4);
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(h0), "r"(h1), "r"(h2), "r"(h3) : "memory");
                    }
                }
            };
            int page = page_of(s0), next_page = page_of(s0 + 1);
            places(page, s0);
            load(p.k, p.k_param, kr, kw);
            load(p.v, p.v_param, vr, vw);
            for (int j = s0; j < s1; ++j, ++step) {
                if (!__all_sync(~0u, wait(sh->k_empty[step & 1], ((step >> 1) & 1) ^ 1, 34))) return false;
                store(base + C::kKAt + (step & 1) * C::kKBytes, kr, kw);
                if (warp == kSoftWarps) {
                    const uint32_t hidden = __ballot_sync(~0u, lane < kStep / 16 && page < 0);
                    if (lane == 0) {
                        sh->unvalued[step & 3] = hidden;
                        ptx::mbar_arrive(ptx::smem_u32(&sh->c_full[step & 3]));
                    }
                }
                ptx::fence_proxy_async();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh->k_full[step & 1]));
                const int after = page_of(j + 2);
                if (j + 1 < s1) {
                    places(next_page, j + 1);
                    load(p.k, p.k_param, kr, kw);
                }
                if (!__all_sync(~0u, wait(sh->v_empty[step & 1], ((step >> 1) & 1) ^ 1, 35))) return false;
                store(base + C::kVAt + (step & 1) * C::kKBytes, vr, vw);
                ptx::fence_proxy_async();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh->v_full[step & 1]));
                if (j + 1 < s1) load(p.v, p.v_param, vr, vw);
                page = next_page, next_page = after;
            }
            return true;
        });
    } else if (warp >= kSoftWarps) {  // ---- unpack keys and values of 8 bits
        constexpr int kPieces = kD / 16;            // 16-byte pieces per token, and passes per step
        constexpr int kPassRows = 128 / kPieces;    // tokens per pass
        const int thread = tid - 32 * kSoftWarps, c = thread % kPieces, r = thread / kPieces;
        uint32_t step = 0;
        for_parts([&](const Unit& u, int head, int s0, int s1) {
            const int32_t* table = p.table + (int64_t)u.b * p.ld_table;
            auto page_of = [&](int j) {  // lanes below 8: page of their 16 tokens of step j, -1 where there is none
                const int tok = u.lo + j * kStep + 16 * lane;
                int page = -1;
                if (j < s1 && lane < kStep / 16 && tok < u.end && tok + 16 > u.first) {
                    page = table[tok >> p.page_log2];
                    if (page < 0 || page >= p.n_pages) page = -1;
                }
                return page;
            };
            uint4 kr[kPieces], vr[kPieces];
            uint32_t at[kPieces];  // of the pieces of a step, in units of 16 bytes; ~0 where there is nothing
            auto places = [&](int pages, int j) {
                const int place = (u.lo + j * kStep) & ((1 << p.page_log2) - 1);
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    const int row = i * kPassRows + r, page = __shfl_sync(~0u, pages, row >> 4);
                    const uint32_t block = (uint32_t)(page * p.heads + head) << p.page_log2;
                    at[i] = page < 0 ? ~0u : (block + ((place + row) & ((1 << p.page_log2) - 1))) * kPieces + c;
                }
            };
            auto load = [&](const int8_t* pool, uint4 (&x)[kPieces]) {
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    x[i] = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);  // becomes -128: finite, under a weight of 0
                    if (at[i] != ~0u) x[i] = __ldg(reinterpret_cast<const uint4*>(pool) + at[i]);
                }
            };
            auto store = [&](uint32_t to, uint4 (&x)[kPieces]) {
                const int swap = (kPieces == 8 ? c >> 2 : 0) & 1;  // the two blocks' threads write opposite halves first: no bank twice
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    const int row = i * kPassRows + r;
                    if (swap) x[i] = make_uint4(x[i].z, x[i].w, x[i].x, x[i].y);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t w0 = (half ? x[i].z : x[i].x) ^ 0x80808080u, w1 = (half ? x[i].w : x[i].y) ^ 0x80808080u;
                        const uint32_t at = to + (c >> 2) * kStep * 128 + row * 128 + ((((2 * c + (half ^ swap)) & 7) ^ (row & 7)) << 4);
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(bytes_to_half2(w0, 0x4140)), "r"(bytes_to_half2(w0, 0x4342)),
                                     "r"(bytes_to_half2(w1, 0x4140)), "r"(bytes_to_half2(w1, 0x4342))
                                     : "memory");
                    }
                }
            };
            auto constants_of = [&](int pages) {  // lanes below 8: scales of their group
                float ks = 0.0f, vs = 0.0f;
                if (pages >= 0) {
                    const int64_t at = (int64_t)pages * p.heads + head;
                    ks = p.k_scale[at], vs = p.v_scale[at];
                }
                return make_float2(ks, vs);
            };
            int page = page_of(s0), next_page = page_of(s0 + 1);
            float2 scale = constants_of(page);
            places(page, s0);
            load(p.k, kr);
            load(p.v, vr);
            for (int j = s0; j < s1; ++j, ++step) {
                if (!__all_sync(~0u, wait(sh->k_empty[step & 1], ((step >> 1) & 1) ^ 1, 34))) return false;
                store(base + C::kKAt + (step & 1) * C::kKBytes, kr);
                if (warp == kSoftWarps) {
                    const bool valued = page >= 0 && scale.y != 0.0f;
                    const uint32_t unvalued = __ballot_sync(~0u, page >= 0 && scale.y == 0.0f);  // lanes that have no tokens have no page
                    if (lane < kStep / 16) sh->constants[step & 3][lane] = make_float4(scale.x, valued ? log2f(scale.y) : -INFINITY, valued ? kDivisorUnit / scale.y : 0.0f, 0.0f);
                    if (lane == 0) sh->unvalued[step & 3] = unvalued;
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh->c_full[step & 3]));
                }
                ptx::fence_proxy_async();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh->k_full[step & 1]));
                const int after = page_of(j + 2);
                const float2 next_scale = constants_of(next_page);
                if (j + 1 < s1) {
                    places(next_page, j + 1);
                    load(p.k, kr);
                }
                if (!__all_sync(~0u, wait(sh->v_empty[step & 1], ((step >> 1) & 1) ^ 1, 35))) return false;
                store(base + C::kVAt + (step & 1) * C::kKBytes, vr);
                ptx::fence_proxy_async();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh->v_full[step & 1]));
                if (j + 1 < s1) load(p.v, vr);
                page = next_page, next_page = after, scale = next_scale;
            }
            return true;
        });
    } else {  // ---- softmax: a thread per query row
        const int t = warp >> 2, row = tid & 127;
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
        uint32_t step = 0, done = 0;  // all steps; steps of this tile
        for_parts([&](const Unit& u, int head, int s0, int s1) {
            if (128 * t >= u.rows) {  // nothing of this tile
                step += s1 - s0;
                return true;
            }
            const int r = u.row0 + 128 * t + row;
            const bool live = 128 * t + row < u.rows;
            const int query = live ? r / p.group : 0, qh = head * p.group + (live ? r % p.group : 0);
            float cq = p.scale_log2;
            {  // the query row to shared memory; BF16 is scaled by a power of two (query_exponent)
                const T16* src = reinterpret_cast<const T16*>(p.q) + (int64_t)(u.q0 + query) * p.ldq + (int64_t)qh * kD;
                float down = 1.0f;
                const uint32_t flip = cq < 0.0f ? 0x80008000u : 0u;  // a negative factor's sign goes to the query
                cq = fabsf(cq);
                if constexpr (kBf16) {
                    uint32_t m = 0;
                    if (live) {
#pragma unroll
                        for (int i = 0; i < kD / 8; ++i) {
                            const uint4 x = __ldg(reinterpret_cast<const uint4*>(src) + i);
                            m = __vimax3_u16x2(__vimax3_u16x2(m, x.x & 0x7FFF7FFFu, x.y & 0x7FFF7FFFu), x.z & 0x7FFF7FFFu, x.w & 0x7FFF7FFFu);
                        }
                    }
                    const int e = query_exponent((int)(max(m & 0xFFFFu, m >> 16) >> 7));
                    down = power_of_2(15 - e);
                    cq *= power_of_2(e - 15);
                }
#pragma unroll
                for (int i = 0; i < kD / 8; ++i) {
                    uint4 x = make_uint4(0, 0, 0, 0);
                    if (live) x = __ldg(reinterpret_cast<const uint4*>(src) + i);
                    if constexpr (kBf16) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float2 f = Half<true>::unpack((&x.x)[e]);
                            (&x.x)[e] = Half<false>::pack(f.x * down, f.y * down);
                        }
                    }
                    x.x ^= flip, x.y ^= flip, x.z ^= flip, x.w ^= flip;
                    if constexpr (kFour)  // in the codes' order
                        x = make_uint4(__byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632), __byte_perm(x.y, x.w, 0x5410), __byte_perm(x.y, x.w, 0x7632));
                    *reinterpret_cast<uint4*>(smem + C::kQAt + t * C::kQBytes + (i >> 3) * 128 * 128 + row * 128 + (((i & 7) ^ (row & 7)) << 4)) = x;
                }
                ptx::fence_proxy_async();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh->q_full[t]));
            }
            const int64_t place = u.place0 + query;
            int see_hi = p.causal ? (int)min((int64_t)u.ctx, place + 1) : u.ctx;
            const int see_lo = p.window > 0 && place + 1 > p.window ? (int)min(place + 1 - p.window, (int64_t)u.ctx) : 0;
            if (!live || see_hi < 0) see_hi = 0;
            // steps that begin in [all_lo, whole_hi] are seen whole by all rows (their ends may pass 32 bits)
            const int all_lo = __reduce_max_sync(~0u, live ? see_lo : 0), whole_hi = __reduce_min_sync(~0u, live ? see_hi : 0x7FFFFFFF) - kStep;
            float m_ref = -INFINITY, sum = 0.0f, rounding = 0.0f;  // rounding: what the divisor is more than the sum (kRounded)
            const bool few = kRounded && __any_sync(~0u, live && see_hi - see_lo < kFewTokens);
            if constexpr (kFour) cq = factor_of(1.0f, cq);
            else sh->unvalued_sum[128 * t + row] = make_float2(-INFINITY, 0.0f);  // this thread's alone
            for (int j = s0; j < s1; ++j, ++step, ++done) {
                const int tok0 = u.lo + j * kStep;
                // the unpacking warps' constants, and S
                if (!__all_sync(~0u, wait(sh->c_full[step & 3], (step >> 2) & 1, 36) && wait(sh->s_full[t], done & 1, 37))) return false;
                ptx::tc_fence_after();
                const uint32_t no_page = kFour ? sh->unvalued[step & 3] : 0;  // of 8 bits the constants hide such tokens
                const bool cut = tok0 < all_lo || tok0 > whole_hi || no_page;
                auto rescale = [&](float shrink) {  // of O, once the products of the step before are in it
                    if (!__all_sync(~0u, wait(sh->o_done[t], (done - 1) & 1, 38))) return false;
                    ptx::tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < kD; c += 32) {
                        uint32_t o[32];
                        ptx::tmem_ld_32x32(o_at[t] + lanes + c, o);
                        ptx::tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * shrink);
                        ptx::tmem_st_32x32(o_at[t] + lanes + c, o);
                    }
                    return true;
                };
                if constexpr (kFour) {
                    // One pass: P against the reference so far, with the largest score beside it, half a step at a time.  Where a row's passes the
                    // reference by too much (its first step, rarely a later one), the reference moves, by a whole number so that what there is of O
                    // and P follows exactly, and the warp goes over the half once more, which P has not taken the place of yet.
                    float part = 0.0f, part_rounding = 0.0f;
#pragma unroll 1
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t from = s_at[t] + lanes + 64 * half;
                        bool again = true;
#pragma unroll 1
                        for (int pass = 0; again; ++pass) {
                            const bool first = m_ref == -INFINITY;
                            const float m = first ? 0.0f : m_ref;
                            float top = -INFINITY, even = 0.0f, odd = 0.0f;
                            uint32_t pk[32];
                            auto weigh = [&](auto is_cut) {
                                uint32_t v[2][16];
                                ptx::tmem_ld_32x16(from, v[0]);
#pragma unroll
                                for (int g = 0; g < 4; ++g) {
                                    uint32_t(&w)[16] = v[g & 1];
                                    ptx::tmem_wait_ld();
                                    if (g < 3) ptx::tmem_ld_32x16(from + 16 * (g + 1), v[(g + 1) & 1]);
                                    if constexpr (decltype(is_cut)::value) {  // what this row does not see
                                        const int at = tok0 + 64 * half + 16 * g;
                                        int lo = no_page >> (4 * half + g) & 1 ? 16 : see_lo - at, hi = see_hi - at;
                                        // both change here as far as the compiler knows: else it compares them in front of the passes, for every step
                                        asm volatile("" : "+r"(lo), "+r"(hi));
#pragma unroll
                                        for (int e = 0; e < 16; ++e)
                                            if (e < lo || e >= hi) w[e] = 0xFF800000u;
                                    }
#pragma unroll
                                    for (int e = 0; e < 8; ++e) {
                                        const float a = __uint_as_float(w[2 * e]), b = __uint_as_float(w[2 * e + 1]);
                                        top = fmaxf(fmaxf(top, a), b);
                                        const float x = exp2_approx(fmaf(a, cq, -m)), y = exp2_approx(fmaf(b, cq, -m));
                                        even += x, odd += y;
                                        pk[8 * g + e] = Half<false>::pack(x, y);
                                    }
                                }
                            };
                            if (cut) weigh(std::true_type());
                            else weigh(std::false_type());
                            top *= cq;
                            const bool grows = pass == 0 && top > (first ? -INFINITY : m_ref + kMostAbove);  // once: then top is 10 above it
                            again = __any_sync(~0u, grows);
                            if (again) {
                                ptx::tmem_wait_st();  // P of the first half and O may have been stored in this step, and are loaded here
                                const float before = m_ref;
                                if (grows) m_ref = first ? top - kBelow : m_ref + ceilf(top - kBelow - m_ref);
                                const float shrink = first || !grows ? 1.0f : exp2_approx(before - m_ref);
                                sum *= shrink, part *= shrink;
                                if constexpr (kRounded) rounding *= shrink, part_rounding *= shrink;
                                if (j > s0 && __any_sync(~0u, shrink != 1.0f) && !rescale(shrink)) return false;
                                if (half) {
                                    uint32_t before_p[32];
                                    ptx::tmem_ld_32x32(s_at[t] + lanes, before_p);
                                    ptx::tmem_wait_ld();
                                    // by two factors: weights of up to 2^15 stay FP16 numbers under 2^-39, whose nearest FP16 number is 0
                                    const __half2 down = __float2half2_rn(fmaxf(shrink, 1.0f / 65536)), rest = __float2half2_rn(fminf(shrink * 65536.0f, 1.0f));
#pragma unroll
                                    for (int e = 0; e < 32; ++e) before_p[e] = mul2(mul2(before_p[e], down), rest);
                                    ptx::tmem_st_32x32(s_at[t] + lanes, before_p);
                                }
                            } else {
                                part += even + odd;
                                if (kRounded && few) {
                                    float rounded = 0.0f;
#pragma unroll
                                    for (int e = 0; e < 32; ++e) {
                                        const float2 f = Half<false>::unpack(pk[e]);
                                        rounded += f.x + f.y;
                                    }
                                    part_rounding += rounded - (even + odd);
                                }
                                ptx::tmem_st_32x32(s_at[t] + lanes + 32 * half, pk);
                            }
                        }
                    }
                    sum += part;
                    if constexpr (kRounded) rounding += part_rounding;
                } else {
                    // Both passes read S in pieces of 32 tokens, the next on its way meanwhile; 16 tokens share their scales.
                    auto for_pieces = [&](auto f) {
                        uint32_t v[2][32];
                        ptx::tmem_ld_32x32(s_at[t] + lanes, v[0]);
#pragma unroll 1
                        for (int g = 0; g < kStep / 16; g += 4) {
                            ptx::tmem_wait_ld();
                            ptx::tmem_ld_32x32(s_at[t] + lanes + 16 * (g + 2), v[1]);
                            f(g, v[0]);
                            ptx::tmem_wait_ld();
                            if (g + 4 < kStep / 16) ptx::tmem_ld_32x32(s_at[t] + lanes + 16 * (g + 4), v[0]);
                            f(g + 2, v[1]);
                        }
                    };
                    auto hide = [&](int g, uint32_t (&v)[32]) {  // what this row does not see
                        const int lo = see_lo - tok0 - 16 * g, hi = see_hi - tok0 - 16 * g;
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (e < lo || e >= hi) v[e] = 0xFF800000u;
                    };
                    auto factor = [&](const float4& k) { return factor_of(k.x, cq); };
                    float top = -INFINITY;  // the largest exponent: of each piece the largest score decides
                    for_pieces([&](int g, uint32_t (&v)[32]) {
                        if (cut) hide(g, v);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float4 k = sh->constants[step & 3][g + h];
                            float m = __uint_as_float(v[16 * h]);
#pragma unroll
                            for (int e = 1; e < 16; ++e) m = fmaxf(m, __uint_as_float(v[16 * h + e]));
                            top = fmaxf(top, fmaf(m, factor(k), k.y));
                        }
                    });
                    const bool first = m_ref == -INFINITY;
                    const bool grows = top > (first ? -INFINITY : m_ref + kMostAbove);
                    const uint32_t unvalued = sh->unvalued[step & 3];
                    if (__any_sync(~0u, grows || unvalued)) {  // one branch on the way of most steps: with two they take 0.6 % longer
                        if (unvalued) add_unvalued(sh, unvalued, step & 3, s_at[t] + lanes, 128 * t + row, see_lo - tok0, see_hi - tok0, cq);
                        const float before = m_ref;
                        m_ref = fmaxf(m_ref, top - kBelow);
                        const float shrink = first || m_ref == before ? 1.0f : exp2_approx(before - m_ref);
                        sum *= shrink;
                        if (j > s0 && __any_sync(~0u, shrink != 1.0f) && !rescale(shrink)) return false;
                    }
                    // P, over the pieces of S that have been read, and the sum of P / vs
                    const float m = m_ref == -INFINITY ? 0.0f : m_ref;
                    float part = 0.0f;
                    for_pieces([&](int g, uint32_t (&v)[32]) {
                        if (cut) hide(g, v);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float4 k = sh->constants[step & 3][g + h];
                            const float a = factor(k), b = k.y - m;
                            float s0 = 0.0f, s1 = 0.0f;
                            uint32_t pk[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const float x = exp2_approx(fmaf(__uint_as_float(v[16 * h + 2 * e]), a, b)), y = exp2_approx(fmaf(__uint_as_float(v[16 * h + 2 * e + 1]), a, b));
                                s0 += x, s1 += y;
                                pk[e] = Half<false>::pack(x, y);
                            }
                            part = fmaf(s0 + s1, k.z, part);
                            ptx::tmem_st_32x8(s_at[t] + lanes + 8 * (g + h), pk);
                        }
                    });
                    sum += part;
                }
                ptx::tmem_wait_st();
                gemm::release(ptx::smem_u32(&sh->p_full[t]), lane, false);
            }
            // ---- the result, or this part's
            if (!__all_sync(~0u, wait(sh->o_done[t], (done - 1) & 1, 39))) return false;
            ptx::tc_fence_after();
            const bool whole = s0 == 0 && s1 == u.steps;
            const int64_t token = u.q0 + query, part_row = ((int64_t)2 * blockIdx.x + (s0 == 0)) * kRows + 128 * t + row;
            // sum is relative to m_ref + kDivisorLog2; with the other tokens' sum relative to the larger reference
            float m_all = kFour ? m_ref : m_ref + kDivisorLog2, keep = kFour ? 1.0f : kDivisorUnit;  // keep: what brings O to that reference
            if (const float2 own = kFour ? make_float2(0.0f, 0.0f) : sh->unvalued_sum[128 * t + row]; own.y != 0.0f) {
                const float m = fmaxf(m_all, own.x), a = exp2_approx(m_all - m);
                sum = fmaf(sum, a, own.y * exp2_approx(own.x - m));
                keep *= a;
                m_all = m;
            }
            const float inv = sum == 0.0f ? 0.0f : keep / (kRounded ? sum + rounding : sum);
            T16* dst = reinterpret_cast<T16*>(p.out) + token * p.ldo + (int64_t)qh * kD;
#pragma unroll 1
            for (int c = 0; c < kD; c += 32) {
                uint32_t o[32];
                ptx::tmem_ld_32x32(o_at[t] + lanes + c, o);
                ptx::tmem_wait_ld();
                if (!live) continue;
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    float f[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(o[e + (kFour ? 2 * (i & 3) + (i >> 2) : i)]);
                    if (whole) {
                        *reinterpret_cast<uint4*>(dst + c + e) = make_uint4(Half<kBf16>::pack(f[0] * inv, f[1] * inv), Half<kBf16>::pack(f[2] * inv, f[3] * inv),
                                                                            Half<kBf16>::pack(f[4] * inv, f[5] * inv), Half<kBf16>::pack(f[6] * inv, f[7] * inv));
                    } else {
                        float4* to = reinterpret_cast<float4*>(p.part_vec + part_row * kD + c + e);
                        to[0] = make_float4(f[0] * keep, f[1] * keep, f[2] * keep, f[3] * keep);
                        to[1] = make_float4(f[4] * keep, f[5] * keep, f[6] * keep, f[7] * keep);
                    }
                }
            }
            ptx::tc_fence_before();
            if (live) {
                if (!whole) p.part_stat[part_row] = make_float4(m_all, sum, rounding, 0.0f);
                else if (p.lse) p.lse[token * p.heads * p.group + qh] = sum == 0.0f ? -INFINITY : (m_all + log2f(sum)) * 0.69314718056f;
            }
            return true;
        });
    }

    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    if (warp == kMultiplier) ptx::tmem_dealloc(tmem, kTmemCols);
}

// Joins the parts of the units that were cut: one warp per (token, query head).
template <int kD, bool kBf16>
__global__ void __launch_bounds__(128) kv_attention_tc_join_kernel(const TcAttnParams tp) {
    using T16 = typename Half<kBf16>::type;
    const AttnParams& p = tp.a;
    const int lane = threadIdx.x & 31, q_heads = p.heads * p.group;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    grid_wait();
    if (item >= p.T * q_heads) return;
    const int token = (int)(item / q_heads), qh = (int)(item % q_heads);
    int b = 0;  // last request that begins at or before the token
    for (int n = p.B; n > 1;) {
        const int half = n >> 1;
        if (p.q_start[b + half] <= token) b += half;
        n -= half;
    }
    const int q0 = min(max(p.q_start[b], 0), (int)p.T), n = max(min(p.q_start[b + 1], (int)p.T) - q0, 0);
    if (token < q0 || token >= q0 + n) return;
    const int row_all = (token - q0) * p.group + qh % p.group, row = row_all % kRows, tile = tp.tile_base[b] + row_all / kRows;
    if (tile >= tp.tile_base[p.B]) return;
    const int64_t steps = (tp.tile_steps[tile + 1] - tp.tile_steps[tile]) / p.heads;
    const int64_t w0 = tp.tile_steps[tile] + qh / p.group * steps;
    const Deal deal(tp.tile_steps[tp.tile_base[p.B]], p.blocks);
    const int first = deal.block_of(w0), last = deal.block_of(w0 + steps - 1);
    if (first == last) return;  // one block had all of it
    constexpr int kVecs = kD == 64 ? 1 : kD / 128;
    float m = -INFINITY, sum = 0.0f, rounding = 0.0f;
    float4 x[kVecs];
#pragma unroll
    for (auto& v : x) v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int i = first; i <= last; ++i) {
        const int64_t part = ((int64_t)2 * i + (i == first)) * kRows + row;
        const float4 st = p.part_stat[part];
        const float m_new = fmaxf(m, st.x);
        const float a = m == -INFINITY ? (sum == 0.0f ? 0.0f : 1.0f) : exp2_approx(m - m_new);
        const float c = st.x == -INFINITY ? (st.y == 0.0f ? 0.0f : 1.0f) : exp2_approx(st.x - m_new);
        sum = fmaf(sum, a, st.y * c), rounding = fmaf(rounding, a, st.z * c);
        m = m_new;
#pragma unroll
        for (int k = 0; k < kVecs; ++k) {
            const int d = 4 * lane + 128 * k;
            if (d < kD) {
                const float4 y = *reinterpret_cast<const float4*>(p.part_vec + part * kD + d);
                x[k].x = fmaf(x[k].x, a, y.x * c), x[k].y = fmaf(x[k].y, a, y.y * c);
                x[k].z = fmaf(x[k].z, a, y.z * c), x[k].w = fmaf(x[k].w, a, y.w * c);
            }
        }
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / (sum + rounding);
    T16* dst = reinterpret_cast<T16*>(p.out) + (int64_t)token * p.ldo + (int64_t)qh * kD;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
        const int d = 4 * lane + 128 * k;
        if (d < kD)
            *reinterpret_cast<uint2*>(dst + d) =
                make_uint2(Half<kBf16>::pack(x[k].x * inv, x[k].y * inv), Half<kBf16>::pack(x[k].z * inv, x[k].w * inv));
    }
    if (lane == 0 && p.lse) p.lse[(int64_t)token * q_heads + qh] = sum == 0.0f ? -INFINITY : (m + log2f(sum)) * 0.69314718056f;
}

struct Workspace {
    size_t steps, of, base, vec, stat, total;
};
Workspace workspace_of(int blocks, int64_t T, int64_t group, int64_t B, int64_t head_dim) {
    const int64_t tiles = T * group / kRows + B;
    Workspace w;
    w.steps = 0;
    w.of = w.steps + (size_t)round_up((tiles + 1) * 8, 256);
    w.base = w.of + (size_t)round_up(tiles * 8, 256);
    w.vec = w.base + (size_t)round_up((B + 1) * 4, 256);
    w.stat = w.vec + (size_t)2 * blocks * kRows * head_dim * 4;
    w.total = w.stat + (size_t)2 * blocks * kRows * 16;
    return w;
}

template <int kD, bool kBf16, bool kFour>
cudaError_t launch(const TcAttnParams& p, int device, cudaStream_t st) {
    using C = Config<kD>;
    static std::atomic<uint64_t> done{0};
    cudaError_t e = allow_smem(kv_attention_tc_kernel<kD, kBf16, kFour>, C::kSmemBytes, device, done);
    if (e != cudaSuccess) return e;
    if ((e = launch_early(kv_attention_units_kernel, dim3(1), kPlanThreads, 0, st, p)) != cudaSuccess) return e;
    if ((e = launch_early(kv_attention_tc_kernel<kD, kBf16, kFour>, dim3(p.a.blocks), kThreads, C::kSmemBytes, st, p)) != cudaSuccess) return e;
    const int64_t items = p.a.T * p.a.heads * p.a.group;
    return launch_early(kv_attention_tc_join_kernel<kD, kBf16>, dim3((unsigned)((items + 3) / 4)), 128, 0, st, p);
}

}  // namespace

size_t kv_attention_tc_workspace_bytes(awe_ctx* h, int64_t T, int64_t group, int64_t B, int64_t head_dim) {
    return workspace_of(h->sm_count, T, group, B, head_dim).total;
}

awe_status_t kv_attention_tc(awe_ctx* h, AttnParams a, int64_t head_dim, bool bf16, bool four, void* workspace, cudaStream_t st) {
    a.blocks = h->sm_count;
    const Workspace w = workspace_of(a.blocks, a.T, a.group, a.B, head_dim);
    uint8_t* at = (uint8_t*)workspace;
    a.part_vec = (float*)(at + w.vec), a.part_stat = (float4*)(at + w.stat);
    TcAttnParams p = {a, (int64_t*)(at + w.steps), (int2*)(at + w.of), (int32_t*)(at + w.base), (int)(a.T * a.group / kRows + a.B), h->status_dev};
    auto run = [&](auto dim, auto is_four) {
        constexpr int kD = decltype(dim)::value;
        constexpr bool kFour = decltype(is_four)::value;
        return bf16 ? launch<kD, true, kFour>(p, h->device, st) : launch<kD, false, kFour>(p, h->device, st);
    };
    using std::integral_constant;
    const cudaError_t e = head_dim == 64 ? (four ? run(integral_constant<int, 64>(), std::true_type()) : run(integral_constant<int, 64>(), std::false_type()))
                                         : (four ? run(integral_constant<int, 128>(), std::true_type()) : run(integral_constant<int, 128>(), std::false_type()));
    if (e != cudaSuccess) return AWE_ERR_CUDA;
    h->launches += 3;
    return AWE_OK;
}

}  // namespace awe
