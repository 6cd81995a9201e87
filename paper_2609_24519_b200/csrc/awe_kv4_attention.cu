// Attention over the paged 4-bit cache (awe_kv4_attention), for few query rows; prompts go to awe_kv_attention_tc.cu.
//
//   s_j = scale * ks_j (q . K_j),   out = sum_j e^(s_j - m) vs_j V_j / sum_j e^(s_j - m)
//
// with the integers K_j, V_j = code - zero (exact in FP16) and the scales ks_j, vs_j of every token.  How work is dealt out to blocks and
// warps, and that the instruction's rows are tokens (then dimensions) and its columns query rows, is as for the 8-bit cache
// (awe_kv_attention.cu).  Different here:
//
//   - The value's scale goes into the weight as an addition to its exponent, w_j = 2^(s_j / ln 2 + log2 vs_j - m), with m 9 to 15 below the
//     largest such exponent so far, so that w_j rounds to FP16 as well as it can for what it contributes, and the products of all tokens
//     add up in one accumulator.  The divisor is the sum of w_j 2^-log2 vs_j before that rounding.  Where the output is FP16, w_j enters as the sum of
//     two FP16 numbers, itself rounded and what that left, in a second product: rounded once, it adds as much to an output's error as the
//     output's own rounding, and a row that sees one token would not have exactly its values (64 requests of up to 8,192 tokens: 103 us for 97).
//     BF16 outputs round eight times as much themselves.
//   - A key's nibble with its sign bit flipped, u = code + 8, moved to the top of a mantissa, is FP16's subnormal u 2^-18 (or, four bits
//     down, u 2^-22, which the queries make up for), so keys take an instruction a pair and half a shift; the zero point goes off the score,
//     q . K = sum q u - (zero + 8) sum q.  (The instruction lines products up by the exponent that subnormals have, 2^-14: with nibbles at
//     the mantissa's bottom, which saves the shift, the logarithm over one token was off by 1.3e-6 of itself with FP16 queries, now by 3.2e-7.)
//     Both sums are FP32, so where a key's codes are its zero point but for one channel the score keeps what rounding 15 sum |q| leaves: 1e-5 for 256
//     elements of spread 4 and a scale of 1.
//   - m is a whole number, so that it and the exponent of the sum add up exactly in the logarithm.
//   - A value's becomes FP16 by inserting it into the mantissa of 1024 (or, four bits up, 16 of it) and subtracting 1024 and the zero point: taken off
//     behind the sum, which is small where many tokens weigh alike, it would cost bits.
//   - A 32-bit word's eight codes come apart in pairs (0, 4), (1, 5), (2, 6), (3, 7), so queries are laid out in that order once; of two
//     tokens' values the 16-bit halves of their words are put together first, which pairs tokens.
//
// A token and head of dimension 128 is 132 bytes of keys and values; what bounds long contexts is not reading them but the instructions: some 370 a
// warp and 16 tokens, half of them on the ALU pipe (52 % of its rate), 61 % of the issue slots.  64 requests of up to 8,192 tokens, 8 heads of 128, BF16: 97 us for
// 282 MB = 2.9 TB/s (tiles of 16 tokens, keys unpacked like values: 110); 2 of 131,072: 80 us (join by a warp a row: 92).  Four blocks of three
// stages on an SM (121 registers).
#include <cooperative_groups.h>

#include <algorithm>
#include <type_traits>

#include "kv4.cuh"
#include "kv_attention_few.cuh"

namespace cg = cooperative_groups;

namespace awe {
namespace {

using namespace serve;
using namespace attn_few;

constexpr float kNoneSeen = -3.402823466e38f;  // the reference of a row that has seen nothing: the lowest number, and not the -inf of hidden scores
constexpr int kTile = 32;  // tokens of a warp's tile: two pieces of 16, which may lie in two pages
constexpr int kStepTokens = kTile * kWarps;

constexpr int64_t kSharedJoins = 1024;
constexpr int kMostCluster = 8;

template <int kD, int kNT>
struct Config {
    static constexpr int kRows = 8 * kNT;
    static constexpr int kStages = kD == 64 ? 5 : 3;
    static constexpr int kRowBytes = kD / 2, kHalfBytes = 16 * kRowBytes;  // of 16 tokens' keys or values
    static constexpr int kValueAt = 2 * kHalfBytes, kParamAt = 4 * kHalfBytes;  // behind the keys; behind those the words of keys, then of values
    static constexpr int kPageAt = kParamAt + 128, kStageBytes = kPageAt + 16;  // the two pages
    static constexpr int kVecPitch = kD + 4;  // floats
    static constexpr int kRingBytes = kWarps * kStages * kStageBytes;
    static constexpr int kJoinBytes = kWarps * kRows * (kVecPitch + 4) * 4;
    static constexpr int kSmemBytes = kRingBytes > kJoinBytes ? kRingBytes : kJoinBytes;  // one after the other
};

// Byte offset of the 16-byte piece c of token row r inside a tile of 16 tokens: pieces are exchanged within 128-byte lines so that the threads
// of one phase of a load (rows g of keys, rows 2 t and the like of values) hit all banks.
template <int kRowBytes>
__device__ __forceinline__ uint32_t piece_at(int r, int c) {
    if constexpr (kRowBytes == 32) return (r >> 2) * 128 + (((((r & 3) << 1) + c) ^ (((r >> 2) & 1) << 1)) << 4);
    else if constexpr (kRowBytes == 64) return (r >> 1) * 128 + (((((r & 1) << 2) + c) ^ (((r >> 1) & 3) << 1)) << 4);
    else return r * 128 + ((c ^ (r & 7)) << 4);
}

// 16 times the scales of two parameter words, within the format's bounds.
__device__ __forceinline__ float2 scales16(uint32_t words) {
    const __half2 s = __hmin2(__hmax2(__halves2half2(__ushort_as_half(words & 0xFFF0u), __ushort_as_half((words >> 16) & 0xFFF0u)),
                                      __float2half2_rn(16.0f * kKv4LeastScale)), __float2half2_rn(16.0f * kKv4MostScale));
    return __half22float2(s);
}
// zero + 8 of two parameter words.
__device__ __forceinline__ float2 kv4_zeros8(uint32_t words) {
    const uint32_t h = sub2(and_xor(words, 0x000F000Fu, 0x64086408u), 0x64006400u);
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
__device__ __forceinline__ float log2_approx(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t lds16(uint32_t addr) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr));
    return v;
}

// The result of a unit from the warps of a cluster, in whose blocks' shared memory they have left what finish_unit takes.  A block writes some
// of the rows, each warp a quarter of their dimensions: kLanes threads with four each, so that 32 / kLanes of the vectors are read side by
// side, and all of a thread's on their way together.
template <int kD, int kRows, bool kBf16>
__device__ __forceinline__ void finish_cluster(const AttnParams& p, const Request& r, const cg::cluster_group& cluster, float* join_vec, float4* join_stat, int head,
                                               int row0, int n_rows) {
    using T16 = typename Half<kBf16>::type;
    constexpr int kVecPitch = kD + 4, kLanes = kD / (4 * kWarps), kGroups = 32 / kLanes, kEach = kMostCluster * kWarps / kGroups;
    static_assert(kMostCluster * kWarps == 32);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, parts = (int)cluster.num_blocks(), n = parts * kWarps;
    const int d = warp * (kD / kWarps) + 4 * (lane % kLanes), group = lane / kLanes;
    for (int row = (int)cluster.block_rank(); row < n_rows; row += parts) {
        float4 st = make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);  // of the cluster's warp `lane`
        if (lane < n) st = cluster.map_shared_rank(join_stat, lane / kWarps)[lane % kWarps * kRows + row];
        float4 y[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int w = group + kGroups * i;
            y[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (w < n) y[i] = *reinterpret_cast<const float4*>(cluster.map_shared_rank(join_vec, w / kWarps) + (w % kWarps * kRows + row) * kVecPitch + d);
        }
        float m = st.x;
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, k));
        const float c = st.x == -INFINITY ? (st.y == 0.0f ? 0.0f : 1.0f) : exp2_approx(st.x - m);
        float sum = st.y * c;
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) sum += __shfl_xor_sync(~0u, sum, k);
        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const float weight = __shfl_sync(~0u, c, group + kGroups * i);
            x.x = fmaf(y[i].x, weight, x.x), x.y = fmaf(y[i].y, weight, x.y), x.z = fmaf(y[i].z, weight, x.z), x.w = fmaf(y[i].w, weight, x.w);
        }
#pragma unroll
        for (int k = 16; k >= kLanes; k >>= 1) {
            x.x += __shfl_xor_sync(~0u, x.x, k), x.y += __shfl_xor_sync(~0u, x.y, k);
            x.z += __shfl_xor_sync(~0u, x.z, k), x.w += __shfl_xor_sync(~0u, x.w, k);
        }
        const int64_t token = r.q0 + (row0 + row) / p.group;
        const int qh = head * p.group + (row0 + row) % p.group;
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        if (group == 0)
            *reinterpret_cast<uint2*>(reinterpret_cast<T16*>(p.out) + token * p.ldo + (int64_t)qh * kD + d) =
                make_uint2(Half<kBf16>::pack(x.x * inv, x.y * inv), Half<kBf16>::pack(x.z * inv, x.w * inv));
        if (threadIdx.x == 0 && p.lse) p.lse[token * p.heads * p.group + qh] = sum == 0.0f ? -INFINITY : log_sum(m, sum);
    }
}

// kCluster: a cluster of blocks per unit (p.whole), each with a part of its steps; else a block has some steps of some units.
template <int kD, int kNT, bool kBf16, bool kCluster>
__global__ void __launch_bounds__(kThreads, kNT == 1 && kD <= 128 ? 4 : 0) kv4_attention_kernel(const AttnParams p) {
    using C = Config<kD, kNT>;
    using T16 = typename Half<kBf16>::type;
    constexpr int kRows = C::kRows, kSteps16 = kD / 16, kWords = kD / 32;  // kWords: of keys, a thread and token
    constexpr int kParts = kBf16 ? 1 : 2;  // FP16 values that a weight is the sum of
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ Search search;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;

    grid_wait();
    Mine mine;
    const cg::cluster_group cluster = cg::this_cluster();
    const int parts = kCluster ? (int)cluster.num_blocks() : 1;
    if (!find_steps<kRows, kStepTokens>(p, search, mine, kCluster ? (int)blockIdx.x / parts : (int)blockIdx.x)) return;  // the whole cluster
    int b = mine.b;
    int64_t at = mine.at;
    Request r = request_of<kRows, kStepTokens>(p, b);
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * C::kStages * C::kStageBytes;
    float* join_vec = reinterpret_cast<float*>(smem);  // in the ring's place once it is empty
    float4* join_stat = reinterpret_cast<float4*>(join_vec + kWarps * kRows * C::kVecPitch);

    for (int64_t pos = mine.begin; pos < mine.end;) {
        while (pos >= at + (p.whole ? r.units : (int64_t)r.units * r.steps)) {
            at += p.whole ? r.units : (int64_t)r.units * r.steps;
            r = request_of<kRows, kStepTokens>(p, ++b);
        }
        const int unit = p.whole ? (int)(pos - at) : (int)((pos - at) / r.steps);
        int step0 = p.whole ? 0 : (int)((pos - at) % r.steps), step1 = p.whole ? r.steps : (int)min((int64_t)r.steps, step0 + mine.end - pos);
        const int head = unit % p.heads, row0 = unit / p.heads * kRows, n_rows = min(kRows, r.n * p.group - row0);
        const int32_t* table = p.table + (int64_t)b * p.ld_table;
        pos += p.whole ? 1 : step1 - step0;
        if constexpr (kCluster) {
            const int rank = (int)cluster.block_rank();
            step0 = (int)((int64_t)r.steps * rank / parts), step1 = (int)((int64_t)r.steps * (rank + 1) / parts);
        }

        // ---- the query rows, as the matrix instruction's 16 x 8 operand: thread (g, t) holds of row g the dimensions t kD / 4 and
        // following, eight at a time in the order of the codes' pairs
        uint32_t qf[kNT][kSteps16][2];
        float cq[kNT][2];                    // factor of the scores of columns 2t, 2t + 1
        float q_sum[kNT][2];                 // sums of those columns' queries, 2^-22 times
        int see_lo[kNT][2], see_hi[kNT][2];  // tokens [see_lo, see_hi) are visible
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) {
            const int row = row0 + 8 * nt + g;
            const bool live = 8 * nt + g < n_rows;
            const int query = live ? row / p.group : 0, qh = head * p.group + (live ? row % p.group : 0);
            const T16* src = reinterpret_cast<const T16*>(p.q) + (int64_t)(r.q0 + query) * p.ldq + (int64_t)qh * kD + t * (kD / 4);
            float factor = p.scale_log2;
#pragma unroll
            for (int w = 0; w < kWords; ++w) {
                uint4 x = make_uint4(0, 0, 0, 0);
                if (live) x = reinterpret_cast<const uint4*>(src)[w];
                qf[nt][2 * w][0] = __byte_perm(x.x, x.z, 0x5410), qf[nt][2 * w][1] = __byte_perm(x.x, x.z, 0x7632);
                qf[nt][2 * w + 1][0] = __byte_perm(x.y, x.w, 0x5410), qf[nt][2 * w + 1][1] = __byte_perm(x.y, x.w, 0x7632);
            }
            query_to_fp16<kBf16, true>(qf[nt], factor);
            // codes four bits up count 16 times, so their queries are a sixteenth; the sum is that of the FP16 values as they are used
            float total = 0.0f;
#pragma unroll
            for (int i = 0; i < kSteps16; ++i) {
                const float2 f = Half<false>::unpack(qf[nt][i][1]);
                qf[nt][i][1] = Half<false>::pack(f.x * 0.0625f, f.y * 0.0625f);
                const float2 x = Half<false>::unpack(qf[nt][i][0]), y = Half<false>::unpack(qf[nt][i][1]);
                total += (x.x + x.y) + 16.0f * (y.x + y.y);
            }
            total += __shfl_xor_sync(~0u, total, 1);
            total += __shfl_xor_sync(~0u, total, 2);
            total *= 2.384185791015625e-7f;  // 2^-22
            int lo_tok, hi_tok;
            visible(p, r, b, query, live, lo_tok, hi_tok);
#pragma unroll
            for (int j = 0; j < 2; ++j) {  // from the thread that loaded row 2t + j
                cq[nt][j] = __shfl_sync(~0u, factor, (2 * t + j) * 4);
                q_sum[nt][j] = __shfl_sync(~0u, total, (2 * t + j) * 4);
                see_lo[nt][j] = __shfl_sync(~0u, lo_tok, (2 * t + j) * 4);
                see_hi[nt][j] = __shfl_sync(~0u, hi_tok, (2 * t + j) * 4);
            }
        }
        const Sees sees = sees_of<kNT>(see_lo, see_hi, n_rows, t);

        float o[kSteps16][kNT][4];
        float m_ref[kNT][2], sum[kNT][2];
#pragma unroll
        for (int i = 0; i < kSteps16; ++i)
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][nt][j] = 0.0f;
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) {
            m_ref[nt][0] = m_ref[nt][1] = kNoneSeen;
            sum[nt][0] = sum[nt][1] = 0.0f;
        }

        // ---- ring of this warp's tiles
        const int n_tiles = step1 - step0;
        const int tok0 = r.lo + step0 * kStepTokens + warp * kTile;
        auto page_of = [&](int i, int half) {  // page of a half of tile i, -1 where it has none
            const int tok = tok0 + i * kStepTokens + 16 * half;
            if (i >= n_tiles || tok >= sees.any_hi || tok + 16 <= sees.any_lo) return -1;
            const int page = table[tok >> p.page_log2];
            return (unsigned)page < (unsigned)p.n_pages ? page : -1;
        };
        // pieces of 16 tokens lie one behind the other in the pools, a page and head's together
        const int piece_log2 = p.page_log2 - 4, piece_mask = (1 << piece_log2) - 1;
        const int8_t *k_from = p.k + 16 * lane, *v_from = p.v + 16 * lane;
        const uint8_t* param_from = reinterpret_cast<const uint8_t*>(lane < 2 ? p.k_param : p.v_param) + 16 * (lane & 1);
        const uint32_t param_to = C::kParamAt + (lane & 2) * 32 + (lane & 1) * 16;
        uint32_t copy_to[C::kHalfBytes / 512];
#pragma unroll
        for (int j = 0; j < C::kHalfBytes / 512; ++j) copy_to[j] = piece_at<C::kRowBytes>((lane + 32 * j) / (C::kRowBytes / 16), (lane + 32 * j) % (C::kRowBytes / 16));
        uint32_t write_at = ring;
        auto fetch = [&](int i, int page0, int page1) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int page = half ? page1 : page0;
                if (page < 0) continue;
                const uint32_t piece = (uint32_t)((tok0 + i * kStepTokens) >> 4) + half & piece_mask;
                const uint64_t from = ((uint64_t)((uint32_t)page * (uint64_t)p.heads + head) << piece_log2) + piece;
                const int8_t *k_at = k_from + from * C::kHalfBytes, *v_at = v_from + from * C::kHalfBytes;
#pragma unroll
                for (int j = 0; j < C::kHalfBytes / 512; ++j) {
                    const uint32_t dst = write_at + copy_to[j];
                    cp_async16_whole(dst + half * C::kHalfBytes, k_at + 512 * j);
                    cp_async16_whole(dst + C::kValueAt + half * C::kHalfBytes, v_at + 512 * j);
                }
                if (lane < 4) cp_async16_whole(write_at + param_to + 32 * half, param_from + from * 32);
            }
            if (lane == 4) asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(write_at + C::kPageAt), "r"(page0), "r"(page1) : "memory");
            cp_async_commit();
            write_at = write_at + C::kStageBytes == ring + C::kStages * C::kStageBytes ? ring : write_at + C::kStageBytes;
        };
#pragma unroll 1
        for (int i = 0; i < C::kStages - 1; ++i) fetch(i, page_of(i, 0), page_of(i, 1));
        int next_page0 = page_of(C::kStages - 1, 0), next_page1 = page_of(C::kStages - 1, 1);

        // places of what this thread reads of 16 tokens: 8 tokens on is half of their bytes on, which changes nothing in the exchange
        const uint32_t key_at = kD == 64 ? piece_at<32>(g, t >> 1) + 8 * (t & 1) : piece_at<C::kRowBytes>(g, t * (kD / 128));
        const uint32_t key_at2 = kD == 256 ? piece_at<128>(g, 2 * t + 1) : 0;
        const uint32_t in_row = kD == 64 ? 4 * (g & 3) : kD == 128 ? 8 * (g & 1) : 0;
        const uint32_t value_at = piece_at<C::kRowBytes>(2 * t, kD == 64 ? g >> 2 : kD == 128 ? g >> 1 : g) + in_row;
        const uint32_t value_at2 = piece_at<C::kRowBytes>(2 * t + 1, kD == 64 ? g >> 2 : kD == 128 ? g >> 1 : g) + in_row;
        uint32_t read_at = ring;
        for (int i = 0; i < n_tiles; ++i) {
            cp_async_wait<C::kStages - 2>();
            __syncwarp();
            fetch(i + C::kStages - 1, next_page0, next_page1);
            next_page0 = page_of(i + C::kStages, 0), next_page1 = page_of(i + C::kStages, 1);
            const uint32_t stage = read_at;
            const uint2 pages = lds64(stage + C::kPageAt);
            // each lane prepares a token of the 32: its key's scale, 2^22 times for codes that come 2^-22 times (here and not in the queries' factor,
            // which may stand at the end of FP32's range: the sum is brought to its size before that), zero + 8, the exponent that is its value's scale, and that back
            const uint32_t words = lds16(stage + C::kParamAt + 2 * lane) | lds16(stage + C::kParamAt + 64 + 2 * lane) << 16;
            const float2 own_scales = scales16(words);
            const float own_key = own_scales.x * 262144.0f, own_zero = kv4_zeros8(words).x, own_log2 = log2_approx(own_scales.y) - 4.0f,
                        own_back = exp2_approx(-own_log2);
            read_at = read_at + C::kStageBytes == ring + C::kStages * C::kStageBytes ? ring : read_at + C::kStageBytes;
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                if ((int)(part ? pages.y : pages.x) < 0) continue;
                const int tile = tok0 + i * kStepTokens + 16 * part;
                const uint32_t ks_at = stage + part * C::kHalfBytes, vs_at = ks_at + C::kValueAt;
                // what the tile holds, all of it on its way before the first product waits for any: keys of the tokens g, g + 8,
                // values of the thread's kD / 8 dimensions of the tokens 2t, 2t + 1, 2t + 8, 2t + 9
                constexpr int kValueWords = kD / 64;
                uint32_t k[2][kWords], v[4][kValueWords];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if constexpr (kD == 64) {
                        const uint2 x = lds64(ks_at + key_at + j * (C::kHalfBytes / 2));
                        k[j][0] = x.x, k[j][1] = x.y;
                    } else {
#pragma unroll
                        for (int c = 0; c < kD / 128; ++c) {
                            const uint4 x = lds128(ks_at + (c ? key_at2 : key_at) + j * (C::kHalfBytes / 2));
                            k[j][4 * c] = x.x, k[j][4 * c + 1] = x.y, k[j][4 * c + 2] = x.z, k[j][4 * c + 3] = x.w;
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t from = vs_at + (j & 1 ? value_at2 : value_at) + (j >> 1) * (C::kHalfBytes / 2);
                    if constexpr (kD == 64) v[j][0] = lds32(from);
                    else if constexpr (kD == 128) {
                        const uint2 x = lds64(from);
                        v[j][0] = x.x, v[j][1] = x.y;
                    } else {
                        const uint4 x = lds128(from);
                        v[j][0] = x.x, v[j][1] = x.y, v[j][2] = x.z, v[j][3] = x.w;
                    }
                }
                const uint32_t pairs_at = stage + C::kParamAt + 64 + 32 * part + 4 * t;
                const Kv4Zeros vz[2] = {lds32(pairs_at), lds32(pairs_at + 16)};

                // scores of 16 tokens (rows g, g + 8) and the query rows (columns 2t, 2t + 1), in two sums that do not wait for each other
                float s[kNT][4], s_odd[kNT][4];
#pragma unroll
                for (int w = 0; w < kWords; ++w) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t x = h ? k[0][w] >> 6 : k[0][w] << 2, y = h ? k[1][w] >> 6 : k[1][w] << 2;
                        const uint32_t f[4] = {and_xor(x, 0x003C003Cu, 0x00200020u), and_xor(y, 0x003C003Cu, 0x00200020u),
                                               and_xor(x, 0x03C003C0u, 0x02000200u), and_xor(y, 0x03C003C0u, 0x02000200u)};
#pragma unroll
                        for (int nt = 0; nt < kNT; ++nt) {
                            float(&to)[4] = h ? s_odd[nt] : s[nt];
                            if (w == 0) mma_16816_zero<false>(to, f, qf[nt][h][0], qf[nt][h][1]);
                            else mma_16816<false>(to, f, qf[nt][2 * w + h][0], qf[nt][2 * w + h][1]);
                        }
                    }
                }
                float ks[2], kz[2], lv[2], back[2];  // of the tokens g and g + 8
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int from = 16 * part + 8 * j + g;
                    ks[j] = __shfl_sync(~0u, own_key, from), kz[j] = __shfl_sync(~0u, own_zero, from);
                    lv[j] = __shfl_sync(~0u, own_log2, from), back[j] = __shfl_sync(~0u, own_back, from);
                }
                const int tok = tile + g;
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        s[nt][j] = fmaf(fmaf(-kz[j >> 1], q_sum[nt][j & 1], s[nt][j] + s_odd[nt][j]) * ks[j >> 1], cq[nt][j & 1], lv[j >> 1]);
                if (tile < sees.all_lo || tile + 16 > sees.all_hi) {
#pragma unroll
                    for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int at_tok = tok + (j >> 1) * 8;
                            if (at_tok < see_lo[nt][j & 1] || at_tok >= see_hi[nt][j & 1]) s[nt][j] = -INFINITY;
                        }
                }
                bool grows = false;
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt)
                    grows |= fmaxf(s[nt][0], s[nt][2]) > m_ref[nt][0] + kMostAbove || fmaxf(s[nt][1], s[nt][3]) > m_ref[nt][1] + kMostAbove;
                if (__any_sync(~0u, grows)) {
#pragma unroll
                    for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            float m = fmaxf(s[nt][j], s[nt][j + 2]);
                            m = fmaxf(m, __shfl_xor_sync(~0u, m, 4));
                            m = fmaxf(m, __shfl_xor_sync(~0u, m, 8));
                            m = fmaxf(m, __shfl_xor_sync(~0u, m, 16));
                            m = fmaxf(rintf(m - kBelow), m_ref[nt][j]);
                            const float a = m == m_ref[nt][j] ? 1.0f : exp2_approx(m_ref[nt][j] - m);
                            m_ref[nt][j] = m;
                            sum[nt][j] *= a;
#pragma unroll
                            for (int c = 0; c < kSteps16; ++c) o[c][nt][j] *= a, o[c][nt][j + 2] *= a;
                        }
                }
                uint32_t pf[kNT][2], rest[kNT][2];
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const float w0 = exp2_approx(s[nt][2 * half] - m_ref[nt][0]), w1 = exp2_approx(s[nt][2 * half + 1] - m_ref[nt][1]);
                        const uint32_t w = Half<false>::pack(w0, w1);
                        sum[nt][0] = fmaf(w0, back[half], sum[nt][0]);
                        sum[nt][1] = fmaf(w1, back[half], sum[nt][1]);
                        pf[nt][half] = movmatrix_trans(w);  // thread (g, t): row g, tokens 2t, 2t + 1 (+ 8 half)
                        if constexpr (kParts > 1) {
                            const float2 f = Half<false>::unpack(w);
                            rest[nt][half] = movmatrix_trans(Half<false>::pack(w0 - f.x, w1 - f.y));
                        }
                    }

#pragma unroll
                for (int w = 0; w < kValueWords; ++w)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t x = __byte_perm(v[0][w], v[1][w], half ? 0x7632 : 0x5410), y = __byte_perm(v[2][w], v[3][w], half ? 0x7632 : 0x5410);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t x2 = x >> (8 * h), y2 = y >> (8 * h);
                            const uint32_t f[4] = {kv4_low_codes(x2, vz[0]), kv4_high_codes(x2, vz[0]), kv4_low_codes(y2, vz[1]), kv4_high_codes(y2, vz[1])};
#pragma unroll
                            for (int nt = 0; nt < kNT; ++nt) {
                                mma_16816<false>(o[4 * w + 2 * half + h][nt], f, pf[nt][0], pf[nt][1]);
                                if constexpr (kParts > 1) mma_16816<false>(o[4 * w + 2 * half + h][nt], f, rest[nt][0], rest[nt][1]);
                            }
                        }
                    }
            }
        }
        cp_async_wait<0>();
        __syncthreads();

        // ---- join the four warps
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float x = sum[nt][j];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) x += __shfl_xor_sync(~0u, x, d);
                const int row = 8 * nt + 2 * t + j;
                if (g == 0) join_stat[warp * kRows + row] = make_float4(m_ref[nt][j] == kNoneSeen ? -INFINITY : m_ref[nt][j], x, x, 0.0f);
                float* vec = join_vec + (warp * kRows + row) * C::kVecPitch + kD / 8 * g;
#pragma unroll
                for (int c = 0; c < kSteps16; ++c) vec[2 * c] = o[c][nt][j], vec[2 * c + 1] = o[c][nt][j + 2];
            }
        if constexpr (kCluster) {
            cluster.sync();
            finish_cluster<kD, kRows, kBf16>(p, r, cluster, join_vec, join_stat, head, row0, n_rows);
            cluster.sync();  // no block goes on, or leaves, while it is read
        } else {
            __syncthreads();
            finish_unit<kD, kRows, kBf16, true>(p, r, join_vec, join_stat, step0, step1, head, row0, n_rows);
            __syncthreads();
        }
    }
}

// Joins the parts of the units that were cut: kShare warps (of a block's kWarps) for a (token, query head).
template <int kD, int kNT, int kShare, bool kBf16>
__global__ void __launch_bounds__(kThreads) kv4_attention_join_kernel(const AttnParams p) {
    constexpr int kRows = 8 * kNT, kVecs = (kD + 127) / 128;
    using T16 = typename Half<kBf16>::type;
    __shared__ float4 stat[kWarps];
    __shared__ float vec[kWarps][kD];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, share = warp % kShare, q_heads = p.heads * p.group;
    const int64_t item = (int64_t)blockIdx.x * (kWarps / kShare) + warp / kShare;
    grid_wait();
    // the request of the token: last b with q_start[b] <= token
    const int token = (int)min(item / q_heads, p.T - 1), qh = (int)(item % q_heads);
    int b = 0;
    for (int n = p.B; n > 1;) {
        const int half = n >> 1;
        if (p.q_start[b + half] <= token) b += half;
        n -= half;
    }
    const Request r = request_of<kRows, kStepTokens>(p, b);
    const int row_all = (token - r.q0) * p.group + qh % p.group, row = row_all % kRows;
    const int64_t w0 = p.unit_steps[b] + (int64_t)(row_all / kRows * p.heads + qh / p.group) * r.steps, w1 = w0 + r.steps;
    const Deal deal(p.unit_steps[p.B], p.blocks);
    const bool live = item < p.T * q_heads && token >= r.q0 && token < r.q0 + r.n;
    const int first = live ? deal.block_of(w0) : 0, last = live ? deal.block_of(w1 - 1) : 0;
    if (first == last) return;  // one block had all of it (or there is nothing); the same for all warps of an item, and a block has one item or needs no barrier
    // this warp's parts first + share, first + share + kShare, ...: 32 at a time, a lane finding the weight of each
    float m = -INFINITY, sum = 0.0f;
    float4 x[kVecs];
#pragma unroll
    for (auto& v : x) v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int i0 = first + share; i0 <= last; i0 += 32 * kShare) {
        const int i = i0 + lane * kShare;
        float4 st = make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
        if (i <= last) st = p.part_stat[((int64_t)2 * i + (i == first)) * kRows + row];  // the first part is the one that begins the unit
        float m_new = st.x;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) m_new = fmaxf(m_new, __shfl_xor_sync(~0u, m_new, d));
        m_new = fmaxf(m, m_new);
        const float c = st.y == 0.0f ? 0.0f : exp2_approx(st.x - m_new), a = sum == 0.0f ? 0.0f : exp2_approx(m - m_new);
        float part_sum = st.y * c;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) part_sum += __shfl_xor_sync(~0u, part_sum, d);
        sum = fmaf(sum, a, part_sum);
        m = m_new;
#pragma unroll
        for (auto& v : x) v.x *= a, v.y *= a, v.z *= a, v.w *= a;
        const int n = min(32, (last - i0) / kShare + 1);
        constexpr int kAhead = 4;  // on their way together
        for (int j0 = 0; j0 < n; j0 += kAhead) {
            float4 y[kAhead][kVecs];
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
#pragma unroll
                for (int k = 0; k < kVecs; ++k) {
                    const int from = i0 + (j0 + j) * kShare;
                    y[j][k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    if (j0 + j < n && 4 * lane + 128 * k < kD)
                        y[j][k] = *reinterpret_cast<const float4*>(p.part_vec + (((int64_t)2 * from + (from == first)) * kRows + row) * kD + 4 * lane + 128 * k);
                }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const float weight = __shfl_sync(~0u, c, (j0 + j) & 31);
#pragma unroll
                for (int k = 0; k < kVecs; ++k) {
                    x[k].x = fmaf(y[j][k].x, weight, x[k].x), x[k].y = fmaf(y[j][k].y, weight, x[k].y);
                    x[k].z = fmaf(y[j][k].z, weight, x[k].z), x[k].w = fmaf(y[j][k].w, weight, x[k].w);
                }
            }
        }
    }
    if constexpr (kShare > 1) {
        if (lane == 0) stat[warp] = make_float4(m, sum, 0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < kVecs; ++k)
            if (4 * lane + 128 * k < kD) *reinterpret_cast<float4*>(&vec[warp][4 * lane + 128 * k]) = x[k];
        __syncthreads();
        if (warp) return;
        float m_all = -INFINITY;
#pragma unroll
        for (int w = 0; w < kShare; ++w) m_all = fmaxf(m_all, stat[w].x);
        sum = 0.0f;
#pragma unroll
        for (auto& v : x) v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < kShare; ++w) {
            const float c = stat[w].y == 0.0f ? 0.0f : exp2_approx(stat[w].x - m_all);
            sum = fmaf(stat[w].y, c, sum);
#pragma unroll
            for (int k = 0; k < kVecs; ++k)
                if (4 * lane + 128 * k < kD) {
                    const float4 y = *reinterpret_cast<const float4*>(&vec[w][4 * lane + 128 * k]);
                    x[k].x = fmaf(y.x, c, x[k].x), x[k].y = fmaf(y.y, c, x[k].y), x[k].z = fmaf(y.z, c, x[k].z), x[k].w = fmaf(y.w, c, x[k].w);
                }
        }
        m = m_all;
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    T16* dst = reinterpret_cast<T16*>(p.out) + (int64_t)token * p.ldo + (int64_t)qh * kD;
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
        if (const int d = 4 * lane + 128 * k; d < kD)
            *reinterpret_cast<uint2*>(dst + d) = make_uint2(Half<kBf16>::pack(x[k].x * inv, x[k].y * inv), Half<kBf16>::pack(x[k].z * inv, x[k].w * inv));
    if (lane == 0 && p.lse) p.lse[(int64_t)token * q_heads + qh] = sum == 0.0f ? -INFINITY : log_sum(m, sum);
}

template <int kD, int kNT>
constexpr int resident_blocks() {
    return 228 * 1024 / (Config<kD, kNT>::kSmemBytes + 1024 + 256);
}
int blocks_of(int sm_count, int64_t head_dim, int nt) {
    const int per_sm = head_dim == 64 ? (nt == 2 ? resident_blocks<64, 2>() : resident_blocks<64, 1>())
                       : head_dim == 128 ? (nt == 2 ? resident_blocks<128, 2>() : resident_blocks<128, 1>())
                                         : resident_blocks<256, 1>();
    return sm_count * std::min(per_sm, nt == 1 && head_dim <= 128 ? 4 : 3);
}

// Contexts of a few steps a block: a cluster of blocks for each unit joins its parts without a second launch.  More blocks a unit while
// there are two of them an SM at most, two a unit as long as all are resident; at most five steps a block, three where parts would have one
// each.  Returns the blocks of a cluster, 1 for none, and the units.
// 8 heads of 128, one query of 4 heads each, us in parts with a join / in clusters of 2, 4, 8: 1 request of 777 tokens 9.0 / 10.3, 8.2, 7.5; of
// 4,000 10.8 / 23, 14.4, 10.6; of 8,000 12.8 / 40, 23, 14.9; 4 of 2,000 11.9 / 15.0, 10.8, 10.1; 8 of 1,000 12.0 / 11.1, 10.1, 11.7; 16 of 1,000 14.5 /
// 12.8, 13.1, 21; 32 of 1,000 22.8 / 19.4, 24.7, 40; 64 of 500 22.8 / 25.8, 38, 77; 2 of 2,000 with 8 queries 19.8 / 20.8, 14.5, 14.8.
int cluster_parts(const AttnParams& p, int nt, int64_t tokens, int blocks, int sm_count, int64_t& units) {
    if (p.window > 0) tokens = std::min(tokens, p.window + p.T / p.B + kStepTokens);
    const int64_t rows = 8 * nt, steps = (tokens + kStepTokens - 1) / kStepTokens;
    units = std::min(p.T * ((p.group + rows - 1) / rows), (p.T * p.group + p.B * (rows - 1)) / rows) * p.heads;  // at most
    int parts = 1;
    while (parts < kMostCluster && parts < steps && units * parts * 2 <= (parts == 1 ? blocks : 2 * sm_count)) parts *= 2;
    return !p.whole && units * p.B <= kWholeScans && steps <= (units * steps <= blocks ? 3 : 5) * parts ? parts : 1;
}

template <int kD, int kNT, bool kBf16>
cudaError_t launch_attention(const AttnParams& p, int parts, int device, cudaStream_t st) {
    using C = Config<kD, kNT>;
    static std::atomic<uint64_t> done{0}, done_cluster{0};
    if (parts > 1) {
        const cudaError_t e = allow_smem(kv4_attention_kernel<kD, kNT, kBf16, true>, C::kSmemBytes, device, done_cluster);
        if (e != cudaSuccess) return e;
        cudaLaunchAttribute attr[2] = {early_launch_attribute(), cluster_attribute(1)};
        attr[1].val.clusterDim.x = parts, attr[1].val.clusterDim.y = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(p.blocks * parts)), cfg.blockDim = dim3(kThreads), cfg.dynamicSmemBytes = C::kSmemBytes, cfg.stream = st;
        cfg.attrs = attr, cfg.numAttrs = 2;
        return cudaLaunchKernelEx(&cfg, kv4_attention_kernel<kD, kNT, kBf16, true>, p);
    }
    cudaError_t e = allow_smem(kv4_attention_kernel<kD, kNT, kBf16, false>, C::kSmemBytes, device, done);
    if (e != cudaSuccess) return e;
    if ((e = launch_early(kv4_attention_kernel<kD, kNT, kBf16, false>, dim3(p.blocks), kThreads, C::kSmemBytes, st, p)) != cudaSuccess) return e;
    if (p.whole) return cudaSuccess;
    // Few rows have many parts each (one token of 131,072: 74), which a block joins faster than a warp; of many rows most have one or two.
    // Attention and its join, a warp and a block a row, us: 1 token over 131,072 (32 rows) 53.8 and 46.6, 8 over 16,000 (256) 48.0 and 47.4,
    // 32 over 4,096 (1,024) 48.8 and 49.2, 64 over 4,096 (2,048) 82.5 and 85.5, 16 x 8 tokens over 4,096 (4,096) 88.7 and 95.5.
    const int64_t items = p.T * p.heads * p.group;
    if (items <= kSharedJoins) return launch_early(kv4_attention_join_kernel<kD, kNT, kWarps, kBf16>, dim3((unsigned)items), kThreads, 0, st, p);
    return launch_early(kv4_attention_join_kernel<kD, kNT, 1, kBf16>, dim3((unsigned)((items + kWarps - 1) / kWarps)), kThreads, 0, st, p);
}

// The kernel on tcgen05 pays from about 64 query rows per request and head on, and 2^29 products.  32 heads over 8 of 128, few rows' kernel
// and tcgen05's, us: 1 request of 16 tokens over 4,096 (64 rows a head) 23.1 and 26.5, of 32 31.6 and 29.6, of 256 147 and 63;
// 128 over 512 (2^28 products) 23.4 and 27.4, 256 over 512 (2^29) 35.2 and 31.0; 16 requests of 4 tokens over 16,384 152 and 286, of 16
// 528 and 296; 300 tokens over 2,000 with 4 heads over 1 27.3 and 29.2.
bool use_tc(const awe_kv4_cache& cache, int64_t T, int64_t B, int64_t n_q_heads, int64_t group, int64_t tokens, int64_t window) {
    const int64_t head_dim = cache.head_dim;
    if (head_dim > 128 || T * group < 64 * B) return false;
    if (cache.n_pages * cache.n_heads * cache.page_size >= (int64_t)1 << 31) return false;  // its token rows are 32 bits
    if (window > 0) tokens = std::min(tokens, window + T / B + 128);
    return (double)T * n_q_heads * head_dim * tokens >= (double)(1 << 29);
}

}  // namespace
}  // namespace awe

using namespace awe;

extern "C" size_t awe_kv4_attention_workspace_bytes(awe_handle_t h, const awe_kv4_cache* cache, int64_t T, int64_t n_q_heads, int64_t B) {
    if (!h || check_kv4_cache(cache) != AWE_OK || T <= 0 || B <= 0 || n_q_heads <= 0 || n_q_heads % cache->n_heads) return 0;
    size_t most = 0;
    for (int nt = 1; nt <= (cache->head_dim < 256 ? 2 : 1); ++nt)
        most = std::max(most, workspace_of(blocks_of(h->sm_count, cache->head_dim, nt), 8 * nt, cache->head_dim, B).total);
    return std::max(most, kv_attention_tc_workspace_bytes(h, T, n_q_heads / cache->n_heads, B, cache->head_dim));
}

extern "C" awe_status_t awe_kv4_attention(awe_handle_t h, const awe_kv4_cache* cache, const void* q_dev, awe_float_t type, int64_t T,
                                          int64_t n_q_heads, int64_t ldq, const int32_t* q_start_dev, const int32_t* ctx_len_dev,
                                          int64_t B, const int32_t* block_table_dev, int64_t max_pages, int64_t ld_table, float scale,
                                          int causal, int64_t window, void* out_dev, int64_t ldo, float* lse_dev,
                                          void* workspace_dev, size_t workspace_bytes, void* stream) {
    if (!h || T < 0 || B < 0) return AWE_ERR_INVALID_ARG;
    const awe_status_t s = check_kv4_cache(cache);
    if (s != AWE_OK) return s;
    AttnParams p = {};
    bool empty = false;
    const awe_status_t c = attention_params(p, empty, q_dev, type, T, n_q_heads, ldq, q_start_dev, ctx_len_dev, B, block_table_dev, max_pages, ld_table,
                                            scale, causal, window, out_dev, ldo, lse_dev, workspace_dev, cache->n_pages, cache->n_heads,
                                            cache->page_size, cache->head_dim);
    if (c != AWE_OK || empty) return c;
    if (workspace_bytes < awe_kv4_attention_workspace_bytes(h, cache, T, n_q_heads, B)) return AWE_ERR_WORKSPACE;
    p.k = reinterpret_cast<const int8_t*>(cache->k_dev), p.v = reinterpret_cast<const int8_t*>(cache->v_dev);
    p.k_param = cache->k_param_dev, p.v_param = cache->v_param_dev;
    if (use_tc(*cache, T, B, n_q_heads, p.group, max_pages * cache->page_size, p.window))
        return kv_attention_tc(h, p, cache->head_dim, type == AWE_BF16, true, workspace_dev, (cudaStream_t)stream);
    const int nt = row_tiles(T, B, p.group, cache->head_dim);
    const int blocks = blocks_of(h->sm_count, cache->head_dim, nt);
    place_few(p, kStepTokens, blocks, nt, cache->head_dim, max_pages * cache->page_size, workspace_dev);
    int64_t units = 0;
    const int parts = cluster_parts(p, nt, max_pages * cache->page_size, blocks, h->sm_count, units);
    if (parts > 1) p.whole = 1, p.blocks = (int)units;
    auto run = [&](auto dim, auto tiles) {
        constexpr int kD = decltype(dim)::value, kNT = decltype(tiles)::value;
        return type == AWE_BF16 ? launch_attention<kD, kNT, true>(p, parts, h->device, (cudaStream_t)stream)
                                : launch_attention<kD, kNT, false>(p, parts, h->device, (cudaStream_t)stream);
    };
    using std::integral_constant;
    cudaError_t e;
    if (cache->head_dim == 256) e = run(integral_constant<int, 256>(), integral_constant<int, 1>());
    else if (cache->head_dim == 128)
        e = nt == 2 ? run(integral_constant<int, 128>(), integral_constant<int, 2>()) : run(integral_constant<int, 128>(), integral_constant<int, 1>());
    else
        e = nt == 2 ? run(integral_constant<int, 64>(), integral_constant<int, 2>()) : run(integral_constant<int, 64>(), integral_constant<int, 1>());
    if (e != cudaSuccess) return AWE_ERR_CUDA;
    h->launches += p.whole ? 1 : 2;
    return AWE_OK;
}
