// Attention over the paged 8-bit cache (awe_kv_attention).
//
//   s_j = scale * ks_j * (q . K_j),   p_j = exp(s_j - m),   out = sum_j vs_j p_j V_j / sum_j p_j
//
// with the integer rows K_j, V_j of the cache and the scales ks_j, vs_j of their page and head.  An 8-bit integer
// is exact in FP16, so both products run on the 16-bit matrix instruction with FP32 sums, and the scales are
// applied in FP32 behind them: ks to the scores, vs to the product of 16 tokens of one page before it joins the
// running sum.
//
// A unit of work is (request, cache head, 8 * kNT query rows); a row is a (query, query head) pair that reads this
// head, so the query heads of a group share every byte of the cache.  The tokens of a unit are cut into steps of
// 64, 16 for each of four warps; all steps of all units in a row are dealt out evenly to as many blocks as are
// resident, so that ragged requests load the machine evenly.  A block that holds a whole unit writes the result,
// others write their part's (m, sum, vector) and a second kernel joins the parts in the order of the tokens.
//
// Products are transposed (rows of the matrix instruction are tokens, then dimensions; its 8 columns are query
// rows), which wastes the least where a group has few heads.  Each warp keeps its own running maximum and sums.
#include <algorithm>
#include <type_traits>

#include "kv_attention_few.cuh"

namespace awe {
awe_status_t check_kv_cache(const awe_kv_cache* c);

namespace {

using namespace serve;
using namespace attn_few;

constexpr int kStepTokens = 16 * kWarps;

template <int kD, int kNT>
struct Config {
    static constexpr int kRows = 8 * kNT;
    static constexpr int kStages = kD == 64 ? 6 : kD == 128 ? 4 : 3;
    static constexpr int kStageBytes = 2 * 16 * kD + 16;  // 16 tokens of keys and values, their two scales and page
    static constexpr int kVecPitch = kD + 4;              // floats
    static constexpr int kRingBytes = kWarps * kStages * kStageBytes;
    static constexpr int kJoinBytes = kWarps * kRows * (kVecPitch + 4) * 4;
    static constexpr int kSmemBytes = kRingBytes > kJoinBytes ? kRingBytes : kJoinBytes;  // one after the other
};

// Byte offset of the 16-byte piece c of token row r inside a tile of 16 tokens: pieces are exchanged within
// 128-byte lines so that the 8 threads of a 16-byte load phase, or the 16 of an 8-byte one, hit all banks.
template <int kD>
__device__ __forceinline__ uint32_t piece_at(int r, int c) {
    if constexpr (kD == 64) return (r >> 1) * 128 + (((((r & 1) << 2) + c) ^ (((r >> 1) & 3) << 1)) << 4);
    return r * kD + ((c & ~7) << 4) + (((c & 7) ^ (r & 7)) << 4);
}

template <int kD, int kNT, bool kBf16>
__global__ void __launch_bounds__(kThreads) kv_attention_kernel(const AttnParams p) {
    using C = Config<kD, kNT>;
    using T16 = typename Half<kBf16>::type;
    constexpr int kRows = C::kRows, kSteps16 = kD / 16;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ Search search;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;

    grid_wait();
    Mine mine;
    if (!find_steps<kRows, kStepTokens>(p, search, mine, blockIdx.x)) return;
    const int64_t begin = mine.begin, end = mine.end;
    int b = mine.b;
    int64_t at = mine.at;
    Request r = request_of<kRows, kStepTokens>(p, b);
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * C::kStages * C::kStageBytes;
    float* join_vec = reinterpret_cast<float*>(smem);  // in the ring's place once it is empty
    float4* join_stat = reinterpret_cast<float4*>(join_vec + kWarps * kRows * C::kVecPitch);

    for (int64_t pos = begin; pos < end;) {
        while (pos >= at + (p.whole ? r.units : (int64_t)r.units * r.steps)) {
            at += p.whole ? r.units : (int64_t)r.units * r.steps;
            r = request_of<kRows, kStepTokens>(p, ++b);
        }
        const int unit = p.whole ? (int)(pos - at) : (int)((pos - at) / r.steps), step0 = p.whole ? 0 : (int)((pos - at) % r.steps);
        const int step1 = p.whole ? r.steps : (int)min((int64_t)r.steps, step0 + end - pos);
        const int head = unit % p.heads, row0 = unit / p.heads * kRows, n_rows = min(kRows, r.n * p.group - row0);
        const int32_t* table = p.table + (int64_t)b * p.ld_table;
        pos += p.whole ? 1 : step1 - step0;

        // ---- the query rows, as the matrix instruction's 16 x 8 operand: thread (g, t) holds of row g the
        // dimensions whose cache pieces it reads.  BF16 rows are scaled by a power of two (query_exponent).
        uint32_t qf[kNT][kSteps16][2];
        float cq[kNT][2];        // factor of the scores of columns 2t, 2t + 1
        int see_lo[kNT][2], see_hi[kNT][2];  // tokens [see_lo, see_hi) are visible
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) {
            const int row = row0 + 8 * nt + g;
            const bool live = 8 * nt + g < n_rows;
            const int query = live ? row / p.group : 0, qh = head * p.group + (live ? row % p.group : 0);
            const T16* src = reinterpret_cast<const T16*>(p.q) + (int64_t)(r.q0 + query) * p.ldq + (int64_t)qh * kD;
            float factor = p.scale_log2;
            uint32_t raw[kSteps16][2];
#pragma unroll
            for (int c = 0; c < kD / 64; ++c) {
                const int piece = kD == 64 ? t : 8 * (c >> 1) + 2 * t + (c & 1);
                uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
                if (live) {
                    lo = *reinterpret_cast<const uint4*>(src + 16 * piece);
                    hi = *reinterpret_cast<const uint4*>(src + 16 * piece + 8);
                }
                raw[4 * c][0] = lo.x, raw[4 * c][1] = lo.y, raw[4 * c + 1][0] = lo.z, raw[4 * c + 1][1] = lo.w;
                raw[4 * c + 2][0] = hi.x, raw[4 * c + 2][1] = hi.y, raw[4 * c + 3][0] = hi.z, raw[4 * c + 3][1] = hi.w;
            }
            query_to_fp16<kBf16, false>(raw, factor);
#pragma unroll
            for (int i = 0; i < kSteps16; ++i) qf[nt][i][0] = raw[i][0], qf[nt][i][1] = raw[i][1];
            int lo_tok, hi_tok;
            visible(p, r, b, query, live, lo_tok, hi_tok);
#pragma unroll
            for (int j = 0; j < 2; ++j) {  // from the thread that loaded row 2t + j
                cq[nt][j] = __shfl_sync(~0u, factor, (2 * t + j) * 4);
                see_lo[nt][j] = __shfl_sync(~0u, lo_tok, (2 * t + j) * 4);
                see_hi[nt][j] = __shfl_sync(~0u, hi_tok, (2 * t + j) * 4);
            }
        }

        const Sees sees = sees_of<kNT>(see_lo, see_hi, n_rows, t);
        const int all_lo = sees.all_lo, all_hi = sees.all_hi, any_lo = sees.any_lo, any_hi = sees.any_hi;

        float o[kSteps16][kNT][4];
        float m_ref[kNT][2], sum[kNT][2], sum_lse[kNT][2];
#pragma unroll
        for (int i = 0; i < kSteps16; ++i)
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][nt][j] = 0.0f;
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) {
            m_ref[nt][0] = m_ref[nt][1] = -INFINITY;
            sum[nt][0] = sum[nt][1] = sum_lse[nt][0] = sum_lse[nt][1] = 0.0f;
        }

        // ---- ring of this warp's 16-token tiles
        const int n_tiles = step1 - step0;
        const int tok0 = r.lo + step0 * kStepTokens + warp * 16;
        auto page_of = [&](int i) {  // page of tile i, -1 where it has none
            const int tok = tok0 + i * kStepTokens;
            if (i >= n_tiles || tok >= any_hi || tok + 16 <= any_lo) return -1;
            const int page = table[tok >> p.page_log2];
            return (unsigned)page < (unsigned)p.n_pages ? page : -1;
        };
        // tiles of 16 tokens lie one behind the other in the pools, a page and head's together
        const int tile_log2 = p.page_log2 - 4, tile_mask = (1 << tile_log2) - 1;
        const int8_t *k_from = p.k + 16 * lane, *v_from = p.v + 16 * lane;
        const float* scale_from = lane == 0 ? p.k_scale : p.v_scale;
        uint32_t write_at = ring;
        auto fetch = [&](int i, int page) {
            if (page >= 0) {
                const uint32_t block = (uint32_t)page * p.heads + head;
                const uint64_t off = (uint64_t)((block << tile_log2) + (((tok0 + i * kStepTokens) >> 4) & tile_mask)) * (16 * kD);
                const int8_t *k_at = k_from + off, *v_at = v_from + off;
#pragma unroll
                for (int j = 0; j < kD / 32; ++j) {
                    const int c = lane + 32 * j;
                    const uint32_t dst = write_at + piece_at<kD>(c / (kD / 16), c % (kD / 16));
                    cp_async16_whole(dst, k_at + 512 * j);
                    cp_async16_whole(dst + 16 * kD, v_at + 512 * j);
                }
                if (lane < 2) cp_async4(write_at + 32 * kD + 4 * lane, scale_from + block);
            }
            if (lane == 2) asm volatile("st.shared.b32 [%0], %1;" ::"r"(write_at + 32 * kD + 8), "r"(page) : "memory");
            cp_async_commit();
            write_at = write_at + C::kStageBytes == ring + C::kStages * C::kStageBytes ? ring : write_at + C::kStageBytes;
        };
#pragma unroll 1
        for (int i = 0; i < C::kStages - 1; ++i) fetch(i, page_of(i));
        int next_page = page_of(C::kStages - 1);

        uint32_t read_at = ring;
        for (int i = 0; i < n_tiles; ++i) {
            cp_async_wait<C::kStages - 2>();
            __syncwarp();
            fetch(i + C::kStages - 1, next_page);
            next_page = page_of(i + C::kStages);
            const uint32_t ks_at = read_at, vs_at = ks_at + 16 * kD;
            read_at = read_at + C::kStageBytes == ring + C::kStages * C::kStageBytes ? ring : read_at + C::kStageBytes;
            if ((int)lds32(ks_at + 32 * kD + 8) < 0) continue;
            const float ks = __uint_as_float(lds32(ks_at + 32 * kD)), vs = __uint_as_float(lds32(ks_at + 32 * kD + 4));

            // what the tile holds, all of it on its way before the first product waits for any: keys of the tokens g, g + 8,
            // values of the thread's kD / 8 dimensions of the tokens 2t, 2t + 1, 2t + 8, 2t + 9
            constexpr int kValueParts = kD == 256 ? 2 : 1, kWords = kD == 64 ? 2 : 4;
            uint4 ka[kD / 64], kb[kD / 64];
            uint32_t v[kValueParts][4][kWords];
#pragma unroll
            for (int c = 0; c < kD / 64; ++c) {
                const int piece = kD == 64 ? t : 8 * (c >> 1) + 2 * t + (c & 1);
                ka[c] = lds128(ks_at + piece_at<kD>(g, piece)), kb[c] = lds128(ks_at + piece_at<kD>(g + 8, piece));
            }
#pragma unroll
            for (int c = 0; c < kValueParts; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int row = 2 * t + (j & 1) + 8 * (j >> 1);
                    if constexpr (kD == 64) {
                        const uint2 x = lds64(vs_at + piece_at<kD>(row, g >> 1) + 8 * (g & 1));
                        v[c][j][0] = x.x, v[c][j][1] = x.y;
                    } else {
                        const uint4 x = lds128(vs_at + piece_at<kD>(row, g + 8 * c));
                        v[c][j][0] = x.x, v[c][j][1] = x.y, v[c][j][2] = x.z, v[c][j][3] = x.w;
                    }
                }

            // scores of 16 tokens (rows g, g + 8) and the query rows (columns 2t, 2t + 1), in two sums that do not wait for each other
            float s[kNT][4], s_odd[kNT][4];
#pragma unroll
            for (int c = 0; c < kD / 64; ++c) {
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint32_t x = flip_signs((&ka[c].x)[w]), y = flip_signs((&kb[c].x)[w]);
                    const uint32_t f[4] = {bytes_to_half2(x, 0x4140), bytes_to_half2(y, 0x4140), bytes_to_half2(x, 0x4342),
                                           bytes_to_half2(y, 0x4342)};
#pragma unroll
                    for (int nt = 0; nt < kNT; ++nt) {
                        float(&to)[4] = w & 1 ? s_odd[nt] : s[nt];
                        if (c == 0 && w < 2) mma_16816_zero<false>(to, f, qf[nt][w][0], qf[nt][w][1]);
                        else mma_16816<false>(to, f, qf[nt][4 * c + w][0], qf[nt][4 * c + w][1]);
                    }
                }
            }
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[nt][j] += s_odd[nt][j];

            const int tile = tok0 + i * kStepTokens, tok = tile + g;
            uint32_t pf[kNT][2];
            bool grows = false;
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt) {
                const float c0 = ks * cq[nt][0], c1 = ks * cq[nt][1];
                s[nt][0] *= c0, s[nt][1] *= c1, s[nt][2] *= c0, s[nt][3] *= c1;
            }
            if (tile < all_lo || tile + 16 > all_hi) {
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int at_tok = tok + (j >> 1) * 8;
                        if (at_tok < see_lo[nt][j & 1] || at_tok >= see_hi[nt][j & 1]) s[nt][j] = -INFINITY;
                    }
            }
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
                        m = fmaxf(m - kBelow, m_ref[nt][j]);
                        const float a = m == m_ref[nt][j] ? 1.0f : exp2_approx(m_ref[nt][j] - m);
                        m_ref[nt][j] = m;
                        sum[nt][j] *= a;
                        sum_lse[nt][j] *= a;
#pragma unroll
                        for (int k = 0; k < kSteps16; ++k) o[k][nt][j] *= a, o[k][nt][j + 2] *= a;
                    }
            }
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const float m0 = m_ref[nt][0] == -INFINITY ? 0.0f : m_ref[nt][0], m1 = m_ref[nt][1] == -INFINITY ? 0.0f : m_ref[nt][1];
                    const float p0 = exp2_approx(s[nt][2 * half] - m0), p1 = exp2_approx(s[nt][2 * half + 1] - m1);
                    const uint32_t w = Half<false>::pack(p0, p1);
                    // The divisor is the sum of the rounded values, so that the rounding cancels where one token
                    // dominates; the logarithm takes the sum of the others.
                    sum_lse[nt][0] += p0;
                    sum_lse[nt][1] += p1;
                    const float2 f = Half<false>::unpack(w);
                    sum[nt][0] += f.x;
                    sum[nt][1] += f.y;
                    pf[nt][half] = movmatrix_trans(w);  // thread (g, t): row g, tokens 2t, 2t + 1 (+ 8 half)
                }

#pragma unroll
            for (int c = 0; c < kValueParts; ++c) {
#pragma unroll
                for (int w = 0; w < kWords; ++w) {
                    const uint32_t x0 = flip_signs(v[c][0][w]), x1 = flip_signs(v[c][1][w]), y0 = flip_signs(v[c][2][w]), y1 = flip_signs(v[c][3][w]);
#pragma unroll
                    for (int pair = 0; pair < 2; ++pair) {
                        const uint32_t sel = pair ? 0x7362 : 0x5140;
                        const uint32_t x = __byte_perm(x0, x1, sel), y = __byte_perm(y0, y1, sel);
                        const uint32_t f[4] = {bytes_to_half2(x, 0x4140), bytes_to_half2(x, 0x4342), bytes_to_half2(y, 0x4140),
                                               bytes_to_half2(y, 0x4342)};
                        const int tile = (c * kWords + w) * 2 + pair;
#pragma unroll
                        for (int nt = 0; nt < kNT; ++nt) {
                            float d[4];
                            mma_16816_zero<false>(d, f, pf[nt][0], pf[nt][1]);
#pragma unroll
                            for (int j = 0; j < 4; ++j) o[tile][nt][j] = fmaf(d[j], vs, o[tile][nt][j]);
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
                float x = sum[nt][j], y = sum_lse[nt][j];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) x += __shfl_xor_sync(~0u, x, d), y += __shfl_xor_sync(~0u, y, d);
                const int row = 8 * nt + 2 * t + j;
                if (g == 0) join_stat[warp * kRows + row] = make_float4(m_ref[nt][j], x, y, 0.0f);
                float* vec = join_vec + (warp * kRows + row) * C::kVecPitch;
#pragma unroll
                for (int k = 0; k < kSteps16; ++k) {
                    // local dimension 2k of this thread's kD / 8, in pieces g (and g + 8)
                    const int dim = kD == 256 ? 128 * (k >> 3) + 16 * g + 2 * (k & 7) : kD / 8 * g + 2 * k;
                    vec[dim] = o[k][nt][j];
                    vec[dim + 1] = o[k][nt][j + 2];
                }
            }
        __syncthreads();
        finish_unit<kD, kRows, kBf16>(p, r, join_vec, join_stat, step0, step1, head, row0, n_rows);
        __syncthreads();
    }
}

// Joins the parts of the units that were cut: one warp per (token, query head).
template <int kD, int kNT, bool kBf16>
__global__ void __launch_bounds__(kThreads) kv_attention_join_kernel(const AttnParams p) {
    constexpr int kRows = 8 * kNT;
    using T16 = typename Half<kBf16>::type;
    const int lane = threadIdx.x & 31, q_heads = p.heads * p.group;
    const int64_t item = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    grid_wait();
    if (item >= p.T * q_heads) return;
    const int token = (int)(item / q_heads), qh = (int)(item % q_heads);
    // the request of the token: last b with q_start[b] <= token
    int b = 0;
    for (int n = p.B; n > 1;) {
        const int half = n >> 1;
        if (p.q_start[b + half] <= token) b += half;
        n -= half;
    }
    const Request r = request_of<kRows, kStepTokens>(p, b);
    if (token < r.q0 || token >= r.q0 + r.n) return;
    const int64_t total = p.unit_steps[p.B];
    const int row_all = (token - r.q0) * p.group + qh % p.group, row = row_all % kRows;
    const int unit = row_all / kRows * p.heads + qh / p.group;
    const int64_t w0 = p.unit_steps[b] + (int64_t)unit * r.steps, w1 = w0 + r.steps;
    const Deal deal(total, p.blocks);
    const int first = deal.block_of(w0), last = deal.block_of(w1 - 1);
    if (first == last) return;  // one block had all of it
    float m = -INFINITY, sum = 0.0f, sum_lse = 0.0f;
    float4 x[kD / 128 + (kD < 128)];
#pragma unroll
    for (auto& v : x) v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int i = first; i <= last; ++i) {
        const int64_t part = ((int64_t)2 * i + (i == first)) * kRows + row;  // the first part is the one that begins the unit
        const float4 st = p.part_stat[part];
        const float m_new = fmaxf(m, st.x);
        const float a = m == -INFINITY ? (sum == 0.0f ? 0.0f : 1.0f) : exp2_approx(m - m_new);
        const float c = st.x == -INFINITY ? (st.y == 0.0f ? 0.0f : 1.0f) : exp2_approx(st.x - m_new);
        sum = fmaf(sum, a, st.y * c);
        sum_lse = fmaf(sum_lse, a, st.z * c);
        m = m_new;
#pragma unroll
        for (int k = 0; k < (int)(sizeof(x) / sizeof(x[0])); ++k) {
            const int d = 4 * lane + 128 * k;
            if (d < kD) {
                const float4 y = *reinterpret_cast<const float4*>(p.part_vec + part * kD + d);
                x[k].x = fmaf(x[k].x, a, y.x * c), x[k].y = fmaf(x[k].y, a, y.y * c);
                x[k].z = fmaf(x[k].z, a, y.z * c), x[k].w = fmaf(x[k].w, a, y.w * c);
            }
        }
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    T16* dst = reinterpret_cast<T16*>(p.out) + (int64_t)token * p.ldo + (int64_t)qh * kD;
#pragma unroll
    for (int k = 0; k < (int)(sizeof(x) / sizeof(x[0])); ++k) {
        const int d = 4 * lane + 128 * k;
        if (d < kD)
            *reinterpret_cast<uint2*>(dst + d) =
                make_uint2(Half<kBf16>::pack(x[k].x * inv, x[k].y * inv), Half<kBf16>::pack(x[k].z * inv, x[k].w * inv));
    }
    if (lane == 0 && p.lse) p.lse[(int64_t)token * q_heads + qh] = sum_lse == 0.0f ? -INFINITY : (m + log2f(sum_lse)) * 0.69314718056f;
}

// tcgen05 pays from about 64 query rows per request and head on, where the work fills its units of 256 rows x 128
// tokens.  us of the kernel for few rows / on tcgen05, 8 heads of 128: one request of 4,096 tokens, 64 rows 28 / 28, 128 rows 40 / 31,
// 1,024 rows 177 / 65; of 512 tokens, 512 rows 25 / 29, 1,024 rows 43 / 32; 16 requests of 16,384 tokens, 16 rows 186 / 334, 64 rows
// 678 / 340.  Of 4,096 tokens each, one request of 2,048 queries among 63 of one: 1,279 / 635; one of 512 among 255: 1,003 / 1,628; one
// of 512 among 63: 504 / 476 (the rule takes the first).  Over 572 sizes of equal requests the rule is 0.5 % above the better of the two, at the worst 1.5 times (one head, one request).  The host knows
// the tokens only by the table's width, and a request's rows by their mean.
bool use_tc(const awe_kv_cache& cache, int64_t T, int64_t B, int64_t n_q_heads, int64_t group, int64_t tokens, int64_t window) {
    const int64_t head_dim = cache.head_dim;
    if (head_dim > 128 || T * group < 64 * B) return false;
    if (cache.n_pages * cache.n_heads * cache.page_size * head_dim >= (int64_t)15 << 32) return false;  // its offsets are 32 bits of 16-byte units
    if (window > 0) tokens = std::min(tokens, window + T / B + 128);
    return (double)T * n_q_heads * head_dim * tokens >= (double)(1 << 29);
}

template <int kD, int kNT>
constexpr int resident_blocks() {
    return 228 * 1024 / (Config<kD, kNT>::kSmemBytes + 1024 + 256);
}
int blocks_of(int sm_count, int64_t head_dim, int nt) {
    const int per_sm = head_dim == 64 ? (nt == 2 ? resident_blocks<64, 2>() : resident_blocks<64, 1>())
                       : head_dim == 128 ? (nt == 2 ? resident_blocks<128, 2>() : resident_blocks<128, 1>())
                                         : resident_blocks<256, 1>();
    return sm_count * std::min(per_sm, 3);
}

template <int kD, int kNT, bool kBf16>
cudaError_t launch_attention(const AttnParams& p, int device, cudaStream_t st) {
    using C = Config<kD, kNT>;
    static std::atomic<uint64_t> done{0};
    cudaError_t e = allow_smem(kv_attention_kernel<kD, kNT, kBf16>, C::kSmemBytes, device, done);
    if (e != cudaSuccess) return e;
    if ((e = launch_early(kv_attention_kernel<kD, kNT, kBf16>, dim3(p.blocks), kThreads, C::kSmemBytes, st, p)) != cudaSuccess) return e;
    if (p.whole) return cudaSuccess;
    const int64_t items = p.T * p.heads * p.group;
    return launch_early(kv_attention_join_kernel<kD, kNT, kBf16>, dim3((unsigned)((items + kWarps - 1) / kWarps)), kThreads, 0, st, p);
}

}  // namespace

awe_status_t attention_params(AttnParams& p, bool& empty, const void* q_dev, awe_float_t type, int64_t T, int64_t n_q_heads, int64_t ldq,
                              const int32_t* q_start_dev, const int32_t* ctx_len_dev, int64_t B, const int32_t* block_table_dev,
                              int64_t max_pages, int64_t ld_table, float scale, int causal, int64_t window, void* out_dev, int64_t ldo,
                              float* lse_dev, void* workspace_dev, int64_t n_pages, int64_t n_heads, int64_t page_size, int64_t head_dim) {
    if ((int)type < AWE_F16 || (int)type > AWE_F32 || window < 0 || (window > 0 && !causal)) return AWE_ERR_INVALID_ARG;
    if (!is_half_type(type)) return AWE_ERR_UNSUPPORTED;
    empty = T == 0 || B == 0;
    if (empty) return AWE_OK;
    const int64_t width = n_q_heads * head_dim;
    if (!q_dev || !q_start_dev || !ctx_len_dev || !block_table_dev || !out_dev || !workspace_dev || n_q_heads <= 0 || n_q_heads % n_heads ||
        max_pages <= 0 || ld_table < max_pages || (T > 1 && (ldq < width || ldo < width)))
        return AWE_ERR_INVALID_ARG;
    if (B > AWE_KV_MAX_REQUESTS || n_q_heads > 65535 || T > INT32_MAX / n_q_heads || max_pages > INT32_MAX / page_size) return AWE_ERR_UNSUPPORTED;
    if ((uintptr_t)q_dev % 16 || (uintptr_t)out_dev % 16 || ldq % 8 || ldo % 8 || (uintptr_t)workspace_dev % 256 ||
        (uintptr_t)q_start_dev % 4 || (uintptr_t)ctx_len_dev % 4 || (uintptr_t)block_table_dev % 4 || (uintptr_t)lse_dev % 4)
        return AWE_ERR_ALIGNMENT;
    int page_log2 = 4;
    while ((1 << page_log2) < page_size) ++page_log2;
    p.q = q_dev, p.out = out_dev, p.lse = lse_dev;
    p.q_start = q_start_dev, p.ctx_len = ctx_len_dev, p.table = block_table_dev;
    p.ldq = ldq, p.ldo = ldo, p.ld_table = ld_table, p.T = T;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.B = (int)B, p.heads = (int)n_heads, p.group = (int)(n_q_heads / n_heads), p.page_log2 = page_log2;
    p.n_pages = (int)n_pages, p.max_pages = (int)max_pages, p.causal = causal != 0;
    p.window = std::min(window, (int64_t)INT32_MAX);  // no context is longer, and the sums that a kernel is chosen by stay in 64 bits
    return AWE_OK;
}
}  // namespace awe

using namespace awe;

extern "C" size_t awe_kv_attention_workspace_bytes(awe_handle_t h, const awe_kv_cache* cache, int64_t T, int64_t n_q_heads,
                                                   int64_t B) {
    if (!h || check_kv_cache(cache) != AWE_OK || T <= 0 || B <= 0 || n_q_heads <= 0 || n_q_heads % cache->n_heads) return 0;
    size_t most = 0;
    for (int nt = 1; nt <= (cache->head_dim < 256 ? 2 : 1); ++nt)
        most = std::max(most, workspace_of(blocks_of(h->sm_count, cache->head_dim, nt), 8 * nt, cache->head_dim, B).total);
    return std::max(most, kv_attention_tc_workspace_bytes(h, T, n_q_heads / cache->n_heads, B, cache->head_dim));
}

extern "C" awe_status_t awe_kv_attention(awe_handle_t h, const awe_kv_cache* cache, const void* q_dev, awe_float_t type,
                                         int64_t T, int64_t n_q_heads, int64_t ldq, const int32_t* q_start_dev,
                                         const int32_t* ctx_len_dev, int64_t B, const int32_t* block_table_dev,
                                         int64_t max_pages, int64_t ld_table, float scale, int causal, int64_t window,
                                         void* out_dev, int64_t ldo, float* lse_dev, void* workspace_dev,
                                         size_t workspace_bytes, void* stream) {
    if (!h || T < 0 || B < 0) return AWE_ERR_INVALID_ARG;
    awe_status_t s = check_kv_cache(cache);
    if (s != AWE_OK) return s;
    AttnParams p = {};
    bool empty = false;
    s = attention_params(p, empty, q_dev, type, T, n_q_heads, ldq, q_start_dev, ctx_len_dev, B, block_table_dev, max_pages, ld_table, scale, causal, window,
                         out_dev, ldo, lse_dev, workspace_dev, cache->n_pages, cache->n_heads, cache->page_size, cache->head_dim);
    if (s != AWE_OK || empty) return s;
    if (workspace_bytes < awe_kv_attention_workspace_bytes(h, cache, T, n_q_heads, B)) return AWE_ERR_WORKSPACE;
    p.k = cache->k_dev, p.v = cache->v_dev, p.k_scale = cache->k_scale_dev, p.v_scale = cache->v_scale_dev;
    if (use_tc(*cache, T, B, n_q_heads, p.group, max_pages * cache->page_size, p.window))
        return kv_attention_tc(h, p, cache->head_dim, type == AWE_BF16, false, workspace_dev, (cudaStream_t)stream);
    const int nt = row_tiles(T, B, p.group, cache->head_dim);
    place_few(p, kStepTokens, blocks_of(h->sm_count, cache->head_dim, nt), nt, cache->head_dim, max_pages * cache->page_size, workspace_dev);
    auto run = [&](auto dim, auto tiles) {
        constexpr int kD = decltype(dim)::value, kNT = decltype(tiles)::value;
        return type == AWE_BF16 ? launch_attention<kD, kNT, true>(p, h->device, (cudaStream_t)stream)
                                : launch_attention<kD, kNT, false>(p, h->device, (cudaStream_t)stream);
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
