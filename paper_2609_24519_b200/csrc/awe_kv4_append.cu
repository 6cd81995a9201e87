// Rotates new queries and keys and stores keys and values into the pages of the 4-bit cache (awe_kv4_append), and reads tokens
// back (awe_kv4_read).
//
//   (a, b) -> (a cos - b sin, b cos + a sin);   scale = (hi - lo) / 15 rounded up to 7 bits,  below = round(lo / scale),
//   nibble ^ 8 = clamp(round(x / scale) - below, 0, 15),  zero = -8 - below
//
// Every token and head stands alone, so all rows are independent: HBM bounds many tokens, latency few.  A row is
// head_dim / 8 threads with eight elements each.  In the halves' order a thread owns four elements and their four partners, so that it
// needs four cosines and four sines, which it keeps for its rows (heads) of a token; each row is read once and written once.  A block has
// one token's keys, its values or a part of its queries: mixed rows in one block took a quarter of the instructions to tell them apart.
//
// 19,707 tokens of 32 query and 8 cache heads of 128: 98 us for 430 MB = 4.4 TB/s, with 62 % of the issue slots used (a first form of one
// kind of block, a division for each value: 138 us); 64 tokens 3.6 us with the read-back behind it.  Their read-back: 27 us for 102 MB = 3.8 TB/s.
#include <algorithm>
#include <type_traits>

#include "kv4.cuh"

namespace awe {
namespace {

using namespace serve;

constexpr int kThreadsLog2 = 7, kThreads = 1 << kThreadsLog2;
constexpr int kMostRows = 4;  // rows of queries that a thread has on their way at once

struct AppendParams {
    const void *q, *k, *v;
    void* q_out;
    uint8_t *k_codes, *v_codes;
    uint16_t *k_param, *v_param;
    const float* table;
    const int32_t* positions;
    const int64_t* slots;
    int64_t T, ldq, ldk, ldv, ldqo, n_slots, n_positions;
    int q_heads, heads, page_log2, rotary_dim;
};

__device__ __forceinline__ float min_nan(float a, float b) {
    float m;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}
constexpr float kRound = 12582912.0f;  // 1.5 * 2^23: adding it to a smaller number leaves the nearest integer, ties to even, in the low bits

// The codes of a thread's eight values of a row (lane groups of kLanes), as nibbles, and the row's scale and round(lo / scale); all
// threads of a warp take part.  Most rows are finite and inside the ends; the others go the long way, with a division for each value.
// So do values next to a tie: the product with the reciprocal is off by less than 10^-5 (of at most 16), and only there must the
// quotient itself say which way to round.
template <int kLanes>
__device__ __forceinline__ uint32_t quantise8(float (&x)[8], float& scale, int& below) {
    float lo = 0.0f, hi = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) lo = min_nan(lo, x[i]), hi = max_nan(hi, x[i]);
#pragma unroll
    for (int d = 1; d < kLanes; d <<= 1) lo = min_nan(lo, __shfl_xor_sync(~0u, lo, d)), hi = max_nan(hi, __shfl_xor_sync(~0u, hi, d));
    bool whole = lo >= -kKv4MostValue && hi <= kKv4MostValue;
    if (!__all_sync(~0u, whole)) {
        lo = 0.0f, hi = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (x[i] != x[i]) x[i] = 0.0f;
            if (fabsf(x[i]) <= 3.402823466e38f) lo = fminf(lo, x[i]), hi = fmaxf(hi, x[i]);
        }
#pragma unroll
        for (int d = 1; d < kLanes; d <<= 1) lo = fminf(lo, __shfl_xor_sync(~0u, lo, d)), hi = fmaxf(hi, __shfl_xor_sync(~0u, hi, d));
        lo = fmaxf(lo, -kKv4MostValue), hi = fminf(hi, kKv4MostValue);
    }
    const float raw = fmaxf(__fdiv_rn(__fsub_rn(hi, lo), 15.0f), kKv4LeastScale);
    scale = __uint_as_float((__float_as_uint(raw) + 0x1FFFFu) & ~0x1FFFFu);  // up to 7 significant bits
    const float inverse = __frcp_rn(scale);
    const float lowest = __fmul_rn(lo, inverse);
    below = (int)rintf(fabsf(lowest - rintf(lowest)) > 0.49999f ? __fdiv_rn(lo, scale) : lowest);
    const int base = __float_as_int(kRound) + below;
    uint32_t u[8];
    float off = whole ? 0.0f : 1.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = __fmul_rn(x[i], inverse), t = __fadd_rn(q, kRound);
        off = fmaxf(off, fabsf(__fsub_rn(q, __fsub_rn(t, kRound))));
        u[i] = (uint32_t)min(__float_as_int(t) - base, 15);
    }
    if (off > 0.49999f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = (uint32_t)fminf(fmaxf(rintf(__fdiv_rn(x[i], scale)) - (float)below, 0.0f), 15.0f);
    }
    uint32_t w = u[7];
#pragma unroll
    for (int i = 6; i >= 0; --i) w = w * 16 + u[i];
    return w ^ 0x88888888u;
}

// Pair i is (f[i], f[i + 4]) of eight elements in the halves' order, (f[2 i], f[2 i + 1]) of interleaved ones.  Products and sums are
// rounded one by one, as written above.
template <bool kPairs>
__device__ __forceinline__ void turn8(float (&f)[8], const float4& c, const float4& s) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float &a = f[kPairs ? 2 * i : i], &b = f[kPairs ? 2 * i + 1 : i + 4];
        const float cos = (&c.x)[i], sin = (&s.x)[i], turned = __fsub_rn(__fmul_rn(a, cos), __fmul_rn(b, sin));
        b = __fadd_rn(__fmul_rn(b, cos), __fmul_rn(a, sin));
        a = turned;
    }
}
template <bool kBf16>
__device__ __forceinline__ void unpack8(const uint2& a, const uint2& b, float (&f)[8]) {
    const float2 x = Half<kBf16>::unpack(a.x), y = Half<kBf16>::unpack(a.y), z = Half<kBf16>::unpack(b.x), w = Half<kBf16>::unpack(b.y);
    f[0] = x.x, f[1] = x.y, f[2] = y.x, f[3] = y.y, f[4] = z.x, f[5] = z.y, f[6] = w.x, f[7] = w.y;
}

// grid: (kTokens tokens, keys / values / parts of the queries).  kPairs: interleaved pairs.
template <int kD, bool kBf16, bool kPairs, int kTokens>
__global__ void __launch_bounds__(kThreads) kv4_append_kernel(const AppendParams p) {
    using T16 = typename Half<kBf16>::type;
    constexpr int kLanes = kD / 8, kRowsAtOnce = kThreads / kLanes;
    const int e = threadIdx.x % kLanes, first = threadIdx.x / kLanes, role = blockIdx.y, half = p.rotary_dim / 2;
    const int64_t t0 = (int64_t)blockIdx.x * kTokens;
    grid_wait();
    // element places: four at `at_a` and four at `at_b`
    const bool turns = kPairs ? 8 * e < p.rotary_dim : 4 * e < half;
    const int at_a = !kPairs && turns ? 4 * e : 8 * e, at_b = !kPairs && turns ? 4 * e + half : 8 * e + 4;
    int64_t slot[kTokens];
    int pos[kTokens];
#pragma unroll
    for (int i = 0; i < kTokens; ++i) {
        const bool in = t0 + i < p.T;
        slot[i] = in && role < 2 ? p.slots[t0 + i] : -1, pos[i] = in ? (p.table ? p.positions[t0 + i] : 0) : -1;
        if (pos[i] >= p.n_positions) pos[i] = -1;
        if (pos[i] < 0 || slot[i] >= p.n_slots) slot[i] = -1;
    }
    auto angles = [&](int i, float4& c, float4& s) {
        const float* from = p.table + (int64_t)max(pos[i], 0) * p.rotary_dim + 4 * e;
        c = __ldg(reinterpret_cast<const float4*>(from)), s = __ldg(reinterpret_cast<const float4*>(from + half));
    };
    if (role >= 2) {
        constexpr int kAhead = kTokens < 2 ? kTokens : 2;  // tokens whose rows are on their way together
        const int row0 = (role - 2) * kMostRows * kRowsAtOnce + first;
#pragma unroll
        for (int i0 = 0; i0 < kTokens; i0 += kAhead) {
            uint2 xa[kAhead][kMostRows], xb[kAhead][kMostRows];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (pos[i0 + i] < 0) continue;
                const T16* from = reinterpret_cast<const T16*>(p.q) + (t0 + i0 + i) * p.ldq;
#pragma unroll
                for (int j = 0; j < kMostRows; ++j) {
                    const T16* row = from + min(row0 + j * kRowsAtOnce, p.q_heads - 1) * kD;
                    xa[i][j] = *reinterpret_cast<const uint2*>(row + at_a), xb[i][j] = *reinterpret_cast<const uint2*>(row + at_b);
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (pos[i0 + i] < 0) continue;
                if (turns) {
                    float4 c, s;
                    angles(i0 + i, c, s);
#pragma unroll
                    for (int j = 0; j < kMostRows; ++j) {
                        float f[8];
                        unpack8<kBf16>(xa[i][j], xb[i][j], f);
                        turn8<kPairs>(f, c, s);
                        xa[i][j] = make_uint2(Half<kBf16>::pack(f[0], f[1]), Half<kBf16>::pack(f[2], f[3]));
                        xb[i][j] = make_uint2(Half<kBf16>::pack(f[4], f[5]), Half<kBf16>::pack(f[6], f[7]));
                    }
                }
                T16* to = reinterpret_cast<T16*>(p.q_out) + (t0 + i0 + i) * p.ldqo + row0 * kD;
#pragma unroll
                for (int j = 0; j < kMostRows; ++j)
                    if (row0 + j * kRowsAtOnce < p.q_heads) {
                        T16* row = to + j * kRowsAtOnce * kD;
                        *reinterpret_cast<uint2*>(row + at_a) = xa[i][j], *reinterpret_cast<uint2*>(row + at_b) = xb[i][j];
                    }
            }
        }
        return;
    }
    const T16* from0 = reinterpret_cast<const T16*>(role ? p.v : p.k);
    const int64_t ld = role ? p.ldv : p.ldk;
    uint8_t* codes = role ? p.v_codes : p.k_codes;
    uint16_t* params = role ? p.v_param : p.k_param;
    // quantised by all of a warp together, for the shuffles: some rows stand twice where the heads do not fill the last pass
#pragma unroll 1
    for (int head0 = 0; head0 < p.heads; head0 += kRowsAtOnce) {
        const int head = min(head0 + first, p.heads - 1);
        uint2 xa[kTokens], xb[kTokens];
#pragma unroll
        for (int i = 0; i < kTokens; ++i) {
            if (slot[i] < 0) continue;
            const T16* row = from0 + (t0 + i) * ld + head * kD;
            xa[i] = *reinterpret_cast<const uint2*>(row + at_a), xb[i] = *reinterpret_cast<const uint2*>(row + at_b);
        }
#pragma unroll
        for (int i = 0; i < kTokens; ++i) {
            if (slot[i] < 0) continue;  // the whole block
            float f[8];
            unpack8<kBf16>(xa[i], xb[i], f);
            if (turns && role == 0) {
                float4 c, s;
                angles(i, c, s);
                turn8<kPairs>(f, c, s);
            }
            float scale;
            int below;
            const uint32_t code = quantise8<kLanes>(f, scale, below);
            const int64_t to = ((((slot[i] >> p.page_log2) * p.heads) + head) << p.page_log2) + (slot[i] & ((1 << p.page_log2) - 1));
            if (head0 + first < p.heads) {
                uint8_t* at = codes + to * (kD / 2);
                if (kPairs || !turns) *reinterpret_cast<uint32_t*>(at + at_a / 2) = code;
                else *reinterpret_cast<uint16_t*>(at + at_a / 2) = (uint16_t)code, *reinterpret_cast<uint16_t*>(at + at_b / 2) = (uint16_t)(code >> 16);
                if (e == 0) params[to] = (uint16_t)(__half_as_ushort(__float2half_rn(scale * 16.0f)) | ((uint32_t)(-8 - below) & 15u));
            }
        }
    }
}

struct ReadParams {
    const uint8_t *k_codes, *v_codes;
    const uint16_t *k_param, *v_param;
    void *k, *v;
    const int64_t* slots;
    int64_t T, ldk, ldv, n_slots;
    int heads, page_log2, lanes_log2;  // a token's keys (or values) are spread over 2^lanes_log2 threads, eight elements at a time
};

// grid: (groups of tokens, keys / values)
template <int kD, bool kBf16>
__global__ void __launch_bounds__(kThreads) kv4_read_kernel(const ReadParams p) {
    using T16 = typename Half<kBf16>::type;
    constexpr int kPieces = kD / 8;
    const bool value = blockIdx.y ? true : p.k == nullptr;
    const int lane = threadIdx.x & ((1 << p.lanes_log2) - 1), pieces = p.heads * kPieces;
    const int64_t t = ((int64_t)blockIdx.x << (kThreadsLog2 - p.lanes_log2)) + (threadIdx.x >> p.lanes_log2);
    grid_wait();
    if (t >= p.T) return;
    const int64_t slot = p.slots[t];
    if (slot < 0 || slot >= p.n_slots) return;
    const int64_t row0 = (((slot >> p.page_log2) * p.heads) << p.page_log2) + (slot & ((1 << p.page_log2) - 1));
    const uint8_t* codes = value ? p.v_codes : p.k_codes;
    const uint16_t* params = value ? p.v_param : p.k_param;
    T16* to = reinterpret_cast<T16*>(value ? p.v : p.k) + t * (value ? p.ldv : p.ldk);
#pragma unroll 2
    for (int i = lane; i < pieces; i += 1 << p.lanes_log2) {
        const int64_t row = row0 + ((int64_t)(i / kPieces) << p.page_log2);
        const uint32_t w = reinterpret_cast<const uint32_t*>(codes + row * (kD / 2))[i % kPieces], word = params[row];
        const __half2 scale = __float2half2_rn(kv4_scale(word));
        const Kv4Zeros zero(word | word << 16);
        // pairs (0, 4), (1, 5), (2, 6), (3, 7), which FP16 holds exactly
        const uint32_t a = mul2(kv4_low_codes(w, zero), scale), b = mul2(kv4_high_codes(w, zero), scale);
        const uint32_t c = mul2(kv4_low_codes(w >> 8, zero), scale), d = mul2(kv4_high_codes(w >> 8, zero), scale);
        uint32_t out[4] = {__byte_perm(a, b, 0x5410), __byte_perm(c, d, 0x5410), __byte_perm(a, b, 0x7632), __byte_perm(c, d, 0x7632)};
        if constexpr (kBf16) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 f = Half<false>::unpack(out[j]);
                out[j] = Half<true>::pack(f.x, f.y);
            }
        }
        *reinterpret_cast<uint4*>(to + 8 * i) = make_uint4(out[0], out[1], out[2], out[3]);
    }
}

int log2_of(int64_t x) {
    int l = 0;
    while (((int64_t)1 << l) < x) ++l;
    return l;
}

template <int kD, int kTokens>
cudaError_t launch_append(const AppendParams& p, bool bf16, bool pairs, cudaStream_t st) {
    const int64_t q_rows = kMostRows * (kThreads / (kD / 8));  // of a block
    const dim3 grid((unsigned)((p.T + kTokens - 1) / kTokens), (unsigned)(2 + (p.q_heads + q_rows - 1) / q_rows));
    if (bf16)
        return pairs ? launch_early(kv4_append_kernel<kD, true, true, kTokens>, grid, kThreads, 0, st, p)
                     : launch_early(kv4_append_kernel<kD, true, false, kTokens>, grid, kThreads, 0, st, p);
    return pairs ? launch_early(kv4_append_kernel<kD, false, true, kTokens>, grid, kThreads, 0, st, p)
                 : launch_early(kv4_append_kernel<kD, false, false, kTokens>, grid, kThreads, 0, st, p);
}

}  // namespace
}  // namespace awe

using namespace awe;
using namespace awe::serve;

extern "C" awe_status_t awe_kv4_append(awe_handle_t h, const awe_kv4_cache* cache, const awe_rotary* rotary, awe_float_t type, int64_t T,
                                       int64_t n_q_heads, const void* q_dev, int64_t ldq, const void* k_dev, int64_t ldk,
                                       const void* v_dev, int64_t ldv, const int32_t* positions_dev, const int64_t* slots_dev,
                                       void* q_out_dev, int64_t ldqo, void* stream) {
    if (!h || T < 0 || n_q_heads < 0) return AWE_ERR_INVALID_ARG;
    const awe_status_t s = check_kv4_cache(cache);
    if (s != AWE_OK) return s;
    if ((int)type < AWE_F16 || (int)type > AWE_F32) return AWE_ERR_INVALID_ARG;
    if (!is_half_type(type)) return AWE_ERR_UNSUPPORTED;
    if (rotary && (!rotary->table_dev || rotary->n_positions <= 0 || rotary->dim <= 0 || rotary->dim > cache->head_dim)) return AWE_ERR_INVALID_ARG;
    if (rotary && rotary->dim % 8) return AWE_ERR_UNSUPPORTED;
    if (T == 0) return AWE_OK;
    const int64_t D = cache->head_dim, width = cache->n_heads * D;
    if (!k_dev || !v_dev || !slots_dev || (rotary && !positions_dev) || (T > 1 && (ldk < width || ldv < width))) return AWE_ERR_INVALID_ARG;
    if (n_q_heads && (!q_dev || !q_out_dev || (T > 1 && (ldq < n_q_heads * D || ldqo < n_q_heads * D)) || (q_dev == q_out_dev && ldq != ldqo)))
        return AWE_ERR_INVALID_ARG;
    if (T > INT32_MAX || n_q_heads > 65535) return AWE_ERR_UNSUPPORTED;
    if ((uintptr_t)k_dev % 16 || (uintptr_t)v_dev % 16 || ldk % 8 || ldv % 8 || (uintptr_t)slots_dev % 8 || (uintptr_t)positions_dev % 4 ||
        (n_q_heads && ((uintptr_t)q_dev % 16 || (uintptr_t)q_out_dev % 16 || ldq % 8 || ldqo % 8)) || (rotary && (uintptr_t)rotary->table_dev % 16))
        return AWE_ERR_ALIGNMENT;
    AppendParams p = {};
    p.q = q_dev, p.k = k_dev, p.v = v_dev, p.q_out = q_out_dev;
    p.k_codes = cache->k_dev, p.v_codes = cache->v_dev, p.k_param = cache->k_param_dev, p.v_param = cache->v_param_dev;
    p.positions = positions_dev, p.slots = slots_dev;
    p.n_positions = 1;  // without a table every token has position 0
    if (rotary) p.table = rotary->table_dev, p.n_positions = rotary->n_positions, p.rotary_dim = (int)rotary->dim;
    p.T = T, p.ldq = ldq, p.ldk = ldk, p.ldv = ldv, p.ldqo = ldqo, p.n_slots = cache->n_pages * cache->page_size;
    p.q_heads = (int)n_q_heads, p.heads = (int)cache->n_heads, p.page_log2 = log2_of(cache->page_size);
    const bool bf16 = type == AWE_BF16, pairs = rotary && rotary->interleaved;
    cudaStream_t st = (cudaStream_t)stream;
    // A block takes four tokens, whose rows are on their way together, where there are enough for every SM to have some blocks.
    // One token a block and four, 32 + 2 x 8 heads of 128, us: 300 tokens 4.4 and 6.3, 600 6.2 and 7.5, 1,200 10.4 and 10.3, 2,400 20.1 and 19.9,
    // 10,000 75.8 and 72.6.
    const bool many = T >= 16 * h->sm_count;
    auto run = [&](auto dim) {
        constexpr int kD = decltype(dim)::value;
        return many ? launch_append<kD, 4>(p, bf16, pairs, st) : launch_append<kD, 1>(p, bf16, pairs, st);
    };
    using std::integral_constant;
    const cudaError_t e = D == 64 ? run(integral_constant<int, 64>()) : D == 128 ? run(integral_constant<int, 128>()) : run(integral_constant<int, 256>());
    if (e != cudaSuccess) return AWE_ERR_CUDA;
    h->launches += 1;
    return AWE_OK;
}

extern "C" awe_status_t awe_kv4_read(awe_handle_t h, const awe_kv4_cache* cache, int64_t T, const int64_t* slots_dev, awe_float_t type,
                                     void* k_out_dev, int64_t ldk, void* v_out_dev, int64_t ldv, void* stream) {
    if (!h || T < 0) return AWE_ERR_INVALID_ARG;
    const awe_status_t s = check_kv4_cache(cache);
    if (s != AWE_OK) return s;
    if ((int)type < AWE_F16 || (int)type > AWE_F32) return AWE_ERR_INVALID_ARG;
    if (!is_half_type(type)) return AWE_ERR_UNSUPPORTED;
    if (T == 0 || (!k_out_dev && !v_out_dev)) return AWE_OK;
    const int64_t width = cache->n_heads * cache->head_dim;
    if (!slots_dev || (T > 1 && ((k_out_dev && ldk < width) || (v_out_dev && ldv < width)))) return AWE_ERR_INVALID_ARG;
    if (T > INT32_MAX) return AWE_ERR_UNSUPPORTED;
    if ((uintptr_t)slots_dev % 8 || (uintptr_t)k_out_dev % 16 || (uintptr_t)v_out_dev % 16 || (k_out_dev && ldk % 8) || (v_out_dev && ldv % 8))
        return AWE_ERR_ALIGNMENT;
    ReadParams p = {cache->k_dev, cache->v_dev, cache->k_param_dev, cache->v_param_dev, k_out_dev, v_out_dev, slots_dev, T, ldk, ldv,
                    cache->n_pages * cache->page_size, (int)cache->n_heads, log2_of(cache->page_size), 0};
    p.lanes_log2 = std::min(kThreadsLog2, log2_of(width / 8));
    const int64_t tokens = kThreads >> p.lanes_log2;  // of a block
    const dim3 grid((unsigned)((T + tokens - 1) / tokens), k_out_dev && v_out_dev ? 2 : 1);
    cudaStream_t st = (cudaStream_t)stream;
    auto run = [&](auto dim) {
        constexpr int kD = decltype(dim)::value;
        return type == AWE_BF16 ? launch_early(kv4_read_kernel<kD, true>, grid, kThreads, 0, st, p) : launch_early(kv4_read_kernel<kD, false>, grid, kThreads, 0, st, p);
    };
    using std::integral_constant;
    const cudaError_t e = cache->head_dim == 64    ? run(integral_constant<int, 64>())
                          : cache->head_dim == 128 ? run(integral_constant<int, 128>())
                                                   : run(integral_constant<int, 256>());
    if (e != cudaSuccess) return AWE_ERR_CUDA;
    h->launches += 1;
    return AWE_OK;
}
