// Rotates new queries and keys and stores keys and values into the pages of the 4-bit cache (awe_kv4_append), and reads tokens
// back (awe_kv4_read).
//
//   (a, b) -> (a cos - b sin, b cos + a sin);   scale = (hi - lo) / 15 rounded up to 7 bits,  below = round(lo / scale),
//   nibble ^ 8 = clamp(round(x / scale) - below, 0, 15),  zero = -8 - below
//
// Every token and head stands alone, so all rows are independent: HBM bounds many tokens, latency few.  A row is
// head_dim / 8 threads with eight elements each.  In the halves' order a thread owns four elements and their four partners, so that it
// needs four cosines and four sines, which it keeps for all of its token's rows (heads); each row is read once and written once.
#include <algorithm>

#include "kv4.cuh"

namespace awe {
namespace {

using namespace serve;

constexpr int kThreads = 256;
constexpr int kMostRows = 4;  // rows (heads) a thread has on their way at once

struct AppendParams {
    const void *q, *k, *v;
    void* q_out;
    uint8_t *k_codes, *v_codes;
    uint16_t *k_param, *v_param;
    const float* table;
    const int32_t* positions;
    const int64_t* slots;
    int64_t ldq, ldk, ldv, ldqo, n_slots, n_positions;
    int q_heads, heads, page_log2, rotary_dim, rows_each;
};

// round(x / s), ties to even.  The product with the reciprocal is off by less than 10^-5 where it matters (below 32 in magnitude),
// so only next to a tie does the quotient itself have to say; a division for each value would take most of the kernel's instructions.
__device__ __forceinline__ float rounded_quotient(float x, float s, float inverse) {
    const float q = __fmul_rn(x, inverse);
    float n = rintf(q);
    if (fabsf(q - n) > 0.49999f) n = rintf(__fdiv_rn(x, s));
    return n;
}

// grid: (tokens, parts of a token's rows).  kPairs: interleaved pairs.
template <int kD, bool kBf16, bool kPairs>
__global__ void __launch_bounds__(kThreads) kv4_append_kernel(const AppendParams p) {
    using T16 = typename Half<kBf16>::type;
    constexpr int kLanes = kD / 8, kRowsAtOnce = kThreads / kLanes;
    const int e = threadIdx.x % kLanes, first_row = blockIdx.y * p.rows_each * kRowsAtOnce + threadIdx.x / kLanes;
    const int64_t t = blockIdx.x;
    const int rows = p.q_heads + 2 * p.heads, half = p.rotary_dim / 2;
    grid_wait();
    const int64_t slot = p.slots[t];
    const bool stored = slot >= 0 && slot < p.n_slots;
    // element places: four at `at_a` and four at `at_b`; pair i is (a[i], b[i]), or for interleaved pairs the eight in order
    const bool turns = kPairs ? 8 * e < p.rotary_dim : 4 * e < half;
    const int at_a = !kPairs && turns ? 4 * e : 8 * e, at_b = !kPairs && turns ? 4 * e + half : 8 * e + 4;
    float4 c = make_float4(1.0f, 1.0f, 1.0f, 1.0f), s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (p.table) {
        const int64_t pos = p.positions[t];
        if (pos < 0 || pos >= p.n_positions) return;
        if (turns) {
            const float* from = p.table + pos * p.rotary_dim + 4 * e;
            c = __ldg(reinterpret_cast<const float4*>(from)), s = __ldg(reinterpret_cast<const float4*>(from + half));
        }
    }
    uint2 xa[kMostRows], xb[kMostRows];
    for (int r0 = first_row, done = 0; done < p.rows_each; done += kMostRows, r0 += kMostRows * kRowsAtOnce) {
#pragma unroll
        for (int j = 0; j < kMostRows; ++j) {
            const int row = r0 + j * kRowsAtOnce;
            xa[j] = xb[j] = make_uint2(0, 0);
            if (done + j >= p.rows_each || row >= rows || (row >= p.q_heads && !stored)) continue;
            const T16* from = row < p.q_heads             ? reinterpret_cast<const T16*>(p.q) + t * p.ldq + (int64_t)row * kD
                              : row < p.q_heads + p.heads ? reinterpret_cast<const T16*>(p.k) + t * p.ldk + (int64_t)(row - p.q_heads) * kD
                                                          : reinterpret_cast<const T16*>(p.v) + t * p.ldv + (int64_t)(row - p.q_heads - p.heads) * kD;
            xa[j] = *reinterpret_cast<const uint2*>(from + at_a), xb[j] = *reinterpret_cast<const uint2*>(from + at_b);
        }
#pragma unroll
        for (int j = 0; j < kMostRows; ++j) {
            const int row = r0 + j * kRowsAtOnce;
            if (done + j >= p.rows_each || row - (int)(threadIdx.x % 32) / kLanes >= rows) continue;  // the same for a whole warp
            float2 f[4] = {Half<kBf16>::unpack(xa[j].x), Half<kBf16>::unpack(xa[j].y), Half<kBf16>::unpack(xb[j].x), Half<kBf16>::unpack(xb[j].y)};
            if (turns && row < p.q_heads + p.heads) {
                // products and sums are rounded one by one, as written above
                auto turn = [](float& a, float& b, float cos, float sin) {
                    const float a2 = __fsub_rn(__fmul_rn(a, cos), __fmul_rn(b, sin));
                    b = __fadd_rn(__fmul_rn(b, cos), __fmul_rn(a, sin));
                    a = a2;
                };
                if constexpr (kPairs) {
                    turn(f[0].x, f[0].y, c.x, s.x), turn(f[1].x, f[1].y, c.y, s.y), turn(f[2].x, f[2].y, c.z, s.z), turn(f[3].x, f[3].y, c.w, s.w);
                } else {
                    turn(f[0].x, f[2].x, c.x, s.x), turn(f[0].y, f[2].y, c.y, s.y), turn(f[1].x, f[3].x, c.z, s.z), turn(f[1].y, f[3].y, c.w, s.w);
                }
            }
            if (row < p.q_heads) {
                T16* to = reinterpret_cast<T16*>(p.q_out) + t * p.ldqo + (int64_t)row * kD;
                *reinterpret_cast<uint2*>(to + at_a) = make_uint2(Half<kBf16>::pack(f[0].x, f[0].y), Half<kBf16>::pack(f[1].x, f[1].y));
                *reinterpret_cast<uint2*>(to + at_b) = make_uint2(Half<kBf16>::pack(f[2].x, f[2].y), Half<kBf16>::pack(f[3].x, f[3].y));
            }
            // the row's ends over its kLanes threads; a warp's rows of queries go along where it has others, for the shuffles
            if (row - (int)(threadIdx.x % 32) / kLanes + 32 / kLanes <= p.q_heads) continue;
            float lo = 0.0f, hi = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float& x = i & 1 ? f[i >> 1].y : f[i >> 1].x;
                if (!(fabsf(x) <= 3.402823466e38f)) {
                    if (x != x) x = 0.0f;
                    continue;
                }
                lo = fminf(lo, x), hi = fmaxf(hi, x);
            }
#pragma unroll
            for (int d = 1; d < kLanes; d <<= 1) lo = fminf(lo, __shfl_xor_sync(~0u, lo, d)), hi = fmaxf(hi, __shfl_xor_sync(~0u, hi, d));
            if (row < p.q_heads || row >= rows || !stored) continue;
            lo = fmaxf(lo, -kKv4MostValue), hi = fminf(hi, kKv4MostValue);
            const float raw = fmaxf(__fdiv_rn(__fsub_rn(hi, lo), 15.0f), kKv4LeastScale);
            const float scale = __uint_as_float((__float_as_uint(raw) + 0x1FFFFu) & ~0x1FFFFu);  // up to 7 significant bits
            const float inverse = __frcp_rn(scale), below = rounded_quotient(lo, scale, inverse);
            uint32_t code[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t w = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 y = f[2 * i + (k >> 1)];
                    const float u = fminf(fmaxf(rounded_quotient(k & 1 ? y.y : y.x, scale, inverse) - below, 0.0f), 15.0f);
                    w |= (uint32_t)u << (4 * k);
                }
                code[i] = w ^ 0x8888u;
            }
            const bool value = row >= p.q_heads + p.heads;
            const int head = row - p.q_heads - (value ? p.heads : 0);
            const int64_t to = (((slot >> p.page_log2) * p.heads + head) << p.page_log2) + (slot & ((1 << p.page_log2) - 1));
            uint8_t* codes = (value ? p.v_codes : p.k_codes) + to * (kD / 2);
            if (at_b == at_a + 4) *reinterpret_cast<uint32_t*>(codes + at_a / 2) = code[0] | code[1] << 16;
            else *reinterpret_cast<uint16_t*>(codes + at_a / 2) = (uint16_t)code[0], *reinterpret_cast<uint16_t*>(codes + at_b / 2) = (uint16_t)code[1];
            if (e == 0)
                (value ? p.v_param : p.k_param)[to] =
                    (uint16_t)(__half_as_ushort(__float2half_rn(scale * 16.0f)) | ((uint32_t)(-8 - (int)below) & 15u));
        }
    }
}

struct ReadParams {
    const uint8_t *k_codes, *v_codes;
    const uint16_t *k_param, *v_param;
    void *k, *v;
    const int64_t* slots;
    int64_t ldk, ldv, n_slots, items;  // items: eight elements each, of keys or of values
    int heads, page_log2, dim_log2;
};

template <bool kBf16>
__global__ void __launch_bounds__(kThreads) kv4_read_kernel(const ReadParams p) {
    using T16 = typename Half<kBf16>::type;
    const int64_t item = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const bool value = blockIdx.y ? true : p.k == nullptr;
    grid_wait();
    if (item >= p.items) return;
    const int64_t row = item >> (p.dim_log2 - 3), t = row / p.heads;
    const int e = (int)(item & ((1 << (p.dim_log2 - 3)) - 1)), head = (int)(row - t * p.heads);
    const int64_t slot = p.slots[t];
    if (slot < 0 || slot >= p.n_slots) return;
    const int64_t from = (((slot >> p.page_log2) * p.heads + head) << p.page_log2) + (slot & ((1 << p.page_log2) - 1));
    const uint32_t w = reinterpret_cast<const uint32_t*>((value ? p.v_codes : p.k_codes) + (from << (p.dim_log2 - 1)))[e] ^ 0x88888888u;
    const uint32_t word = (value ? p.v_param : p.k_param)[from];
    const float scale = kv4_scale(word), zero = (float)kv4_zero8(word);
    uint32_t out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        out[i] = Half<kBf16>::pack(((float)((w >> (8 * i)) & 15u) - zero) * scale, ((float)((w >> (8 * i + 4)) & 15u) - zero) * scale);
    T16* to = reinterpret_cast<T16*>(value ? p.v : p.k) + t * (value ? p.ldv : p.ldk) + ((int64_t)head << p.dim_log2) + 8 * e;
    *reinterpret_cast<uint4*>(to) = make_uint4(out[0], out[1], out[2], out[3]);
}

int log2_of(int64_t x) {
    int l = 0;
    while (((int64_t)1 << l) < x) ++l;
    return l;
}

template <int kD>
cudaError_t launch_append(const AppendParams& p, bool bf16, bool pairs, dim3 grid, cudaStream_t st) {
    if (bf16)
        return pairs ? launch_early(kv4_append_kernel<kD, true, true>, grid, kThreads, 0, st, p)
                     : launch_early(kv4_append_kernel<kD, true, false>, grid, kThreads, 0, st, p);
    return pairs ? launch_early(kv4_append_kernel<kD, false, true>, grid, kThreads, 0, st, p)
                 : launch_early(kv4_append_kernel<kD, false, false>, grid, kThreads, 0, st, p);
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
    if (rotary) p.table = rotary->table_dev, p.n_positions = rotary->n_positions, p.rotary_dim = (int)rotary->dim;
    p.ldq = ldq, p.ldk = ldk, p.ldv = ldv, p.ldqo = ldqo, p.n_slots = cache->n_pages * cache->page_size;
    p.q_heads = (int)n_q_heads, p.heads = (int)cache->n_heads, p.page_log2 = log2_of(cache->page_size);
    // A token's rows go to several blocks while there are few tokens, since a block's rows then wait for one another.
    const int64_t at_once = kThreads / (D / 8), passes = (n_q_heads + 2 * cache->n_heads + at_once - 1) / at_once;
    int64_t parts = 1;
    while (parts < passes && T * parts < 4 * h->sm_count) ++parts;
    p.rows_each = (int)((passes + parts - 1) / parts);
    const dim3 grid((unsigned)T, (unsigned)((passes + p.rows_each - 1) / p.rows_each));
    const bool bf16 = type == AWE_BF16, pairs = rotary && rotary->interleaved;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = D == 64    ? launch_append<64>(p, bf16, pairs, grid, st)
                          : D == 128 ? launch_append<128>(p, bf16, pairs, grid, st)
                                     : launch_append<256>(p, bf16, pairs, grid, st);
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
    if (T > INT32_MAX || T * width / 8 / kThreads >= INT32_MAX) return AWE_ERR_UNSUPPORTED;
    if ((uintptr_t)slots_dev % 8 || (uintptr_t)k_out_dev % 16 || (uintptr_t)v_out_dev % 16 || (k_out_dev && ldk % 8) || (v_out_dev && ldv % 8))
        return AWE_ERR_ALIGNMENT;
    ReadParams p = {cache->k_dev, cache->v_dev, cache->k_param_dev, cache->v_param_dev, k_out_dev, v_out_dev, slots_dev, ldk, ldv,
                    cache->n_pages * cache->page_size, T * width / 8, (int)cache->n_heads, log2_of(cache->page_size), log2_of(cache->head_dim)};
    const dim3 grid((unsigned)((p.items + kThreads - 1) / kThreads), k_out_dev && v_out_dev ? 2 : 1);
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = type == AWE_BF16 ? launch_early(kv4_read_kernel<true>, grid, kThreads, 0, st, p)
                                           : launch_early(kv4_read_kernel<false>, grid, kThreads, 0, st, p);
    if (e != cudaSuccess) return AWE_ERR_CUDA;
    h->launches += 1;
    return AWE_OK;
}
