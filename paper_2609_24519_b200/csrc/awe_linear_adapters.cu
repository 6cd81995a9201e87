// Low-rank adapters of many requests beside a shared projection (awe_linear_adapters).
//
//   u = A x (rank sums over K),   y = base + scale * B u (N sums over the rank)
//
// A unit is up to kTokens tokens of one request, and a cluster of blocks computes it in one launch: K is cut over the cluster's
// warps, the parts of u are added in shared memory, over the blocks in distributed shared memory, and then N is cut over the same
// warps.  Both products run on the 16-bit matrix instruction with FP32 sums.  The bytes of x, base, y and the adapters bound many
// tokens, latency few; no operand is read by more than a few flops a byte, so operands go from global memory to registers directly:
// the order of k (and of the rank) inside an instruction is free, and a thread takes eight (four) neighbours of a row.
// u enters the second product as several 16-bit values, the rounded u, the rounded rest of it, and so on: two hold 22 bits in FP16 and 16 in
// BF16, whose third (24 bits) is taken where y is FP32.
//
// One token, 8,192 x 8,192, rank 64: 7.5 us (a cluster of 16); 64 tokens with 48 adapters, 4,096 x 4,096, rank 16: 7.2 us (clusters of 4); 4,096
// tokens of 8 requests, same sizes: 28 us for 101 MB = 3.6 TB/s.  Tried for many tokens without gain: 16 warps a block, tiles of 32 columns with the
// next one's loads under way, results straight from the registers (27 to 30 us; unaligned rows 82 to 102 instead of 69).
//
// Units are numbered without a scan: request b's first is q_start[b] / kTokens + b, which leaves room for all of its units before
// those of request b + 1.  Some numbers have no unit; their clusters end at once.
#include <cooperative_groups.h>

#include <algorithm>
#include <type_traits>

#include "awe_internal.h"
#include "serve_common.cuh"

namespace cg = cooperative_groups;

namespace awe {
namespace {

using namespace serve;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMostCluster = 16;
constexpr int kFew = 8, kMany = 32;  // tokens of a unit

struct AdapterParams {
    const void *a, *b, *x, *base;
    void* y;
    const float* scale;
    const int32_t *q_start, *adapter;
    int64_t ldx, ldb, ldy, n_adapters;
    int T, B, N, K, rank;
    int vec;  // vec: rows of base and y lie on 16 bytes
};

struct Unit {
    int token, n, adapter;  // n = 0: none
};
template <int kTokens>
__device__ __forceinline__ Unit unit_of(const AdapterParams& p, int number) {
    const int lane = threadIdx.x & 31;
    // last request whose first unit is not behind `number`: 32 requests are asked at a time, and the last time all that is wanted of them
    int b = 0;
    for (int n = p.B;;) {
        const int stride = (n + 31) / 32, i = lane * stride;
        int start = 0, next = 0, adapter = -1;
        if (i < n) {
            start = min(max(p.q_start[b + i], 0), p.T);
            if (stride == 1) next = p.q_start[b + i + 1], adapter = p.adapter[b + i];
        }
        const int unit = start / kTokens + b + i;
        const unsigned fits = __ballot_sync(~0u, i < n && unit <= number);
        if (!fits) return {0, 0, -1};
        const int last = 31 - __clz(fits);
        if (stride == 1) {
            const int first = __shfl_sync(~0u, unit, last), q1 = min(__shfl_sync(~0u, next, last), p.T);
            const int64_t token = __shfl_sync(~0u, start, last) + (int64_t)(number - first) * kTokens;
            return {(int)min(token, (int64_t)p.T), (int)max(min((int64_t)kTokens, q1 - token), (int64_t)0), __shfl_sync(~0u, adapter, last)};
        }
        b += last * stride, n = min(stride, n - last * stride);
    }
}

// A pair of values as kParts pairs of 16 bits: the rounded value, the rounded rest, and so on.  FP16's range is narrow, so the values of a
// token are brought below 2^15 first (`down`).
template <bool kBf16, int kParts>
struct Split {
    uint32_t part[kParts];
    __device__ __forceinline__ Split() {}
    __device__ __forceinline__ Split(float x, float y, float down) {
        if constexpr (!kBf16) x *= down, y *= down;
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            part[i] = Half<kBf16>::pack(x, y);
            const float2 f = Half<kBf16>::unpack(part[i]);
            x -= f.x, y -= f.y;
        }
    }
};
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
// Exponent that brings magnitudes up to `largest` below 2^15; both powers of it stay normal.
__device__ __forceinline__ int down_exponent(float largest) { return min(max((int)(__float_as_uint(largest) >> 23) - 127 - 14, -120), 120); }

__device__ __forceinline__ uint4 load16_if(const void* from, bool live) {
    return live ? __ldg(reinterpret_cast<const uint4*>(from)) : make_uint4(0, 0, 0, 0);
}
__device__ __forceinline__ uint2 load8_if(const void* from, bool live) {
    return live ? __ldg(reinterpret_cast<const uint2*>(from)) : make_uint2(0, 0);
}
// Elements of base and y: FP32, or of the adapters' type.
template <bool kBf16, bool kF32>
struct Out {
    using T = typename std::conditional<kF32, float, typename Half<kBf16>::type>::type;
    static __device__ __forceinline__ float load(const T* at) {
        if constexpr (kF32) return *at;
        else return Half<kBf16>::to_float(*at);
    }
    static __device__ __forceinline__ void store(T* at, float y) {
        if constexpr (kF32) *at = y;
        else *at = Half<kBf16>::from_float(y);
    }
};

// A unit without an adapter: y = base, a row a warp, kAhead pieces on their way together (base and y may be one, so the compiler moves no
// load before a store).
template <class O, int kAhead>
__device__ __forceinline__ void copy_base(const AdapterParams& p, const Unit& u, int part, int parts) {
    using T = typename O::T;
    if (p.base == p.y) return;
    constexpr int kPiece = 16 / sizeof(T);
    const int lane = threadIdx.x & 31;
    // few tokens: a row goes to several warps
    const int warps = parts * kWarps, each = max(warps / u.n, 1), warp = part * kWarps + (threadIdx.x >> 5);
    if (warp >= each * u.n && each > 1) return;
    for (int i = warp / each; i < u.n; i += max(warps / each, 1)) {
        const T* from = reinterpret_cast<const T*>(p.base) + (int64_t)(u.token + i) * p.ldb;
        T* to = reinterpret_cast<T*>(p.y) + (int64_t)(u.token + i) * p.ldy;
        const int first = (warp % each) * 32 + lane, stride = 32 * each;
        int done = 0;
        if (p.vec) {
            const int pieces = p.N / kPiece;
            for (int c = first; c < pieces; c += kAhead * stride) {
                uint4 x[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) x[k] = p.base && c + k * stride < pieces ? reinterpret_cast<const uint4*>(from)[c + k * stride] : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int k = 0; k < kAhead; ++k)
                    if (c + k * stride < pieces) reinterpret_cast<uint4*>(to)[c + k * stride] = x[k];
            }
            done = pieces * kPiece;
        }
        for (int n = done + first; n < p.N; n += 2 * kAhead * stride) {
            float x[2 * kAhead];
#pragma unroll
            for (int k = 0; k < 2 * kAhead; ++k) x[k] = p.base && n + k * stride < p.N ? O::load(from + n + k * stride) : 0.0f;
#pragma unroll
            for (int k = 0; k < 2 * kAhead; ++k)
                if (n + k * stride < p.N) O::store(to + n + k * stride, x[k]);
        }
    }
}

// Few tokens: they are the instruction's 8 columns, ranks (then n) its 16 rows.  kRT tiles of 16 ranks.
template <bool kBf16, bool kF32, int kRT>
__global__ void __launch_bounds__(kThreads, kRT == 1 ? 3 : 2) adapters_few_kernel(const AdapterParams p) {
    using T16 = typename Half<kBf16>::type;
    using O = Out<kBf16, kF32>;
    constexpr int kParts = kBf16 && kF32 ? 3 : 2;
    constexpr int kValues = kRT * 16 * kFew;
    constexpr int kAhead = kRT <= 2 ? 4 : (kRT == 4 ? 2 : 1);  // steps of k, and tiles of n, that are on their way together
    __shared__ float sums[kWarps][kValues];
    __shared__ float part_sums[kValues];
    __shared__ float low[kValues];
    cg::cluster_group cluster = cg::this_cluster();
    const int parts = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    grid_wait();
    const Unit u = unit_of<kFew>(p, blockIdx.x / parts);
    if (u.n == 0) return;  // the whole cluster
    if (u.adapter < 0 || u.adapter >= p.n_adapters) return copy_base<O, 4>(p, u, part, parts);
    const int me = part * kWarps + warp, all = parts * kWarps;

    // ---- u = A x
    const T16* a = reinterpret_cast<const T16*>(p.a) + (int64_t)u.adapter * p.rank * p.K;
    const T16* x = reinterpret_cast<const T16*>(p.x) + (int64_t)(u.token + min(g, u.n - 1)) * p.ldx;
    float acc[kRT][4];
#pragma unroll
    for (int r = 0; r < kRT; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[r][i] = 0.0f;
    const int steps = (p.K + 31) / 32;
    for (int s0 = me; s0 < steps; s0 += all * kAhead) {
        uint4 xw[kAhead], aw[kAhead][kRT][2];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int k = (s0 + i * all) * 32 + 8 * t;
            const bool in = s0 + i * all < steps && k < p.K;
            xw[i] = load16_if(x + k, in && g < u.n);
#pragma unroll
            for (int r = 0; r < kRT; ++r)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int row = 16 * r + 8 * j + g;
                    aw[i][r][j] = load16_if(a + (int64_t)row * p.K + k, in && row < p.rank);
                }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int r = 0; r < kRT; ++r) {
                const uint4 &lo = aw[i][r][0], &hi = aw[i][r][1];
                const uint32_t f0[4] = {lo.x, hi.x, lo.y, hi.y}, f1[4] = {lo.z, hi.z, lo.w, hi.w};
                mma_16816<kBf16>(acc[r], f0, xw[i].x, xw[i].y);
                mma_16816<kBf16>(acc[r], f1, xw[i].z, xw[i].w);
            }
    }
    // rows of B and of base for the first tiles of n are fetched while u is put together
    const T16* b = reinterpret_cast<const T16*>(p.b) + (int64_t)u.adapter * p.N * p.rank;
    const int tiles = (p.N + 15) / 16;
    uint2 bw[kAhead][kRT][2];
    float base[kAhead][4];
    const typename O::T* base_row[2];  // of the tokens 2 t, 2 t + 1
    typename O::T* y_row[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        base_row[c] = reinterpret_cast<const typename O::T*>(p.base) + (int64_t)(u.token + 2 * t + c) * p.ldb;
        y_row[c] = reinterpret_cast<typename O::T*>(p.y) + (int64_t)(u.token + 2 * t + c) * p.ldy;
    }
    auto fetch = [&](int tile0) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int tile = tile0 + i * all;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int n = 16 * tile + 8 * j + g;
#pragma unroll
                for (int r = 0; r < kRT; ++r) bw[i][r][j] = load8_if(b + (int64_t)n * p.rank + 16 * r + 4 * t, tile < tiles && n < p.N && 16 * r + 4 * t < p.rank);
#pragma unroll
                for (int c = 0; c < 2; ++c) base[i][2 * j + c] = p.base && tile < tiles && n < p.N && 2 * t + c < u.n ? O::load(base_row[c] + n) : 0.0f;
            }
        }
    };
    fetch(me);
#pragma unroll
    for (int r = 0; r < kRT; ++r)
#pragma unroll
        for (int j = 0; j < 2; ++j) *reinterpret_cast<float2*>(&sums[warp][(16 * r + 8 * j + g) * kFew + 2 * t]) = make_float2(acc[r][2 * j], acc[r][2 * j + 1]);
    __syncthreads();
    for (int i = tid; i < kValues; i += kThreads) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) s += sums[w][i];
        part_sums[i] = s;
    }
    cluster.sync();
    const float scale = p.scale ? p.scale[u.adapter] : 1.0f;
    for (int i = tid; i < kValues; i += kThreads) {
        float s[kMostCluster];
#pragma unroll
        for (int j = 0; j < kMostCluster; ++j) s[j] = j < parts ? cluster.map_shared_rank(part_sums, j)[i] : 0.0f;
        float v = 0.0f;
#pragma unroll
        for (int j = 0; j < kMostCluster; ++j) v += s[j];
        low[i] = v * scale;
    }
    cluster.barrier_arrive();  // this block has read the others' sums
    __syncthreads();

    // ---- y = base + B u: thread (g, t) holds of token g the ranks 4 t .. 4 t + 3 of each tile
    Split<kBf16, kParts> vs[kRT][2];
    float back[2] = {1.0f, 1.0f};  // of the tokens 2 t, 2 t + 1
    {
        float v[kRT][4], most = 0.0f;
#pragma unroll
        for (int r = 0; r < kRT; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[r][i] = low[(16 * r + 4 * t + i) * kFew + g], most = fmaxf(most, fabsf(v[r][i]));
        float down = 1.0f;
        if constexpr (!kBf16) {
            most = fmaxf(most, __shfl_xor_sync(~0u, most, 1));
            most = fmaxf(most, __shfl_xor_sync(~0u, most, 2));
            const int e = down_exponent(most);
            down = power_of_two(-e);
            back[0] = __shfl_sync(~0u, power_of_two(e), 8 * t), back[1] = __shfl_sync(~0u, power_of_two(e), 8 * t + 4);
        }
#pragma unroll
        for (int r = 0; r < kRT; ++r)
#pragma unroll
            for (int i = 0; i < 2; ++i) vs[r][i] = Split<kBf16, kParts>(v[r][2 * i], v[r][2 * i + 1], down);
    }
    for (int tile0 = me; tile0 < tiles; tile0 += all * kAhead) {
        if (tile0 != me) fetch(tile0);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int tile = tile0 + i * all;
            if (tile >= tiles) break;
            float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int r = 0; r < kRT; ++r) {
                const uint32_t f[4] = {bw[i][r][0].x, bw[i][r][1].x, bw[i][r][0].y, bw[i][r][1].y};
#pragma unroll
                for (int k = kParts - 1; k >= 0; --k) mma_16816<kBf16>(d, f, vs[r][0].part[k], vs[r][1].part[k]);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    if (const int n = 16 * tile + 8 * j + g; n < p.N && 2 * t + c < u.n)
                        O::store(y_row[c] + n, fmaf(d[2 * j + c], back[c], base[i][2 * j + c]));
        }
    }
    cluster.barrier_wait();  // no block leaves while its sums are read
}

// Many tokens: 32 of them, in two tiles of the instruction's 16 rows; ranks (then n) are its 8 columns.  kRN tiles of 8 ranks.
template <int kRN>
struct Many {
    static constexpr int kPitch = 8 * kRN + 4;  // floats of a token's sums
    static constexpr int kSumsBytes = kWarps * kMany * kPitch * 4;
    static constexpr int kOutPitch = 64 + 4;
    static constexpr int kOutBytes = kWarps * 16 * kOutPitch * 4;  // in the sums' place once they are added
    static constexpr int kPartAt = kSumsBytes > kOutBytes ? kSumsBytes : kOutBytes;
    static constexpr int kLowAt = kPartAt + kMany * kPitch * 4;
    static constexpr int kSmemBytes = kLowAt + kMany * kPitch * 4;
};

template <bool kBf16, bool kF32, int kRN>
__global__ void __launch_bounds__(kThreads, kRN <= 8 ? 2 : 1) adapters_many_kernel(const AdapterParams p) {
    using M = Many<kRN>;
    using T16 = typename Half<kBf16>::type;
    using O = Out<kBf16, kF32>;
    constexpr int kParts = kBf16 && kF32 ? 3 : 2;
    extern __shared__ __align__(16) uint8_t smem[];
    float* sums = reinterpret_cast<float*>(smem);
    float* part_sums = reinterpret_cast<float*>(smem + M::kPartAt);
    float* low = reinterpret_cast<float*>(smem + M::kLowAt);
    cg::cluster_group cluster = cg::this_cluster();
    const int parts = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    grid_wait();
    const Unit u = unit_of<kMany>(p, blockIdx.x / parts);
    if (u.n == 0) return;  // the whole cluster
    if (u.adapter < 0 || u.adapter >= p.n_adapters) return copy_base<O, 8>(p, u, part, parts);
    const int me = part * kWarps + warp, all = parts * kWarps;

    // ---- u = A x: every warp has all tokens and ranks and its own steps of k
    const T16* a = reinterpret_cast<const T16*>(p.a) + (int64_t)u.adapter * p.rank * p.K;
    const T16* x = reinterpret_cast<const T16*>(p.x) + (int64_t)u.token * p.ldx;
    {
        float acc[2][kRN][4];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int r = 0; r < kRN; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][r][i] = 0.0f;
        const int steps = (p.K + 31) / 32;
        constexpr int kAhead = kRN <= 4 ? 2 : 1;
        for (int s0 = me; s0 < steps; s0 += all * kAhead) {
            uint4 xw[kAhead][4], aw[kAhead][kRN];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int k = (s0 + i * all) * 32 + 8 * t;
                const bool in = s0 + i * all < steps && k < p.K;
#pragma unroll
                for (int j = 0; j < 4; ++j) xw[i][j] = load16_if(x + (8 * j + g) * p.ldx + k, in && 8 * j + g < u.n);
#pragma unroll
                for (int r = 0; r < kRN; ++r) aw[i][r] = load16_if(a + (int64_t)(8 * r + g) * p.K + k, in && 8 * r + g < p.rank);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const uint4 &lo = xw[i][2 * m], &hi = xw[i][2 * m + 1];
                    const uint32_t f0[4] = {lo.x, hi.x, lo.y, hi.y}, f1[4] = {lo.z, hi.z, lo.w, hi.w};
#pragma unroll
                    for (int r = 0; r < kRN; ++r) {
                        mma_16816<kBf16>(acc[m][r], f0, aw[i][r].x, aw[i][r].y);
                        mma_16816<kBf16>(acc[m][r], f1, aw[i][r].z, aw[i][r].w);
                    }
                }
        }
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int r = 0; r < kRN; ++r)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    *reinterpret_cast<float2*>(sums + (warp * kMany + 16 * m + 8 * j + g) * M::kPitch + 8 * r + 2 * t) = make_float2(acc[m][r][2 * j], acc[m][r][2 * j + 1]);
    }
    __syncthreads();
    for (int i = tid; i < kMany * 2 * kRN; i += kThreads) {  // four ranks of a token each
        const int at = i / (2 * kRN) * M::kPitch + i % (2 * kRN) * 4;
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float4 o = *reinterpret_cast<const float4*>(sums + w * kMany * M::kPitch + at);
            s.x += o.x, s.y += o.y, s.z += o.z, s.w += o.w;
        }
        *reinterpret_cast<float4*>(part_sums + at) = s;
    }
    cluster.sync();
    const float scale = p.scale ? p.scale[u.adapter] : 1.0f;
    for (int i = tid; i < kMany * 2 * kRN; i += kThreads) {
        const int at = i / (2 * kRN) * M::kPitch + i % (2 * kRN) * 4;
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int j = 0; j < kMostCluster; ++j) {
            if (j >= parts) break;
            const float4 o = *reinterpret_cast<const float4*>(cluster.map_shared_rank(part_sums, j) + at);
            s.x += o.x, s.y += o.y, s.z += o.z, s.w += o.w;
        }
        *reinterpret_cast<float4*>(low + at) = make_float4(s.x * scale, s.y * scale, s.z * scale, s.w * scale);
    }
    cluster.barrier_arrive();  // this block has read the others' sums
    __syncthreads();

    // ---- y = base + B u: a warp has one tile of 16 tokens and 64 columns of y at a time
    constexpr int kRT = kRN / 2;
    const int m = warp & 1;
    uint32_t vs[kParts][kRT][4];
    float back[2] = {1.0f, 1.0f};  // of the tokens g, g + 8
    {
        const float* from[2] = {low + (16 * m + g) * M::kPitch + 4 * t, low + (16 * m + 8 + g) * M::kPitch + 4 * t};
        float down[2] = {1.0f, 1.0f};
        if constexpr (!kBf16) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float most = 0.0f;
#pragma unroll
                for (int r = 0; r < kRT; ++r) {
                    const float4 v = *reinterpret_cast<const float4*>(from[j] + 16 * r);
                    most = fmaxf(fmaxf(most, fmaxf(fabsf(v.x), fabsf(v.y))), fmaxf(fabsf(v.z), fabsf(v.w)));
                }
                most = fmaxf(most, __shfl_xor_sync(~0u, most, 1));
                most = fmaxf(most, __shfl_xor_sync(~0u, most, 2));
                const int e = down_exponent(most);
                down[j] = power_of_two(-e), back[j] = power_of_two(e);
            }
        }
#pragma unroll
        for (int r = 0; r < kRT; ++r)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float4 v = *reinterpret_cast<const float4*>(from[j] + 16 * r);
                const Split<kBf16, kParts> x(v.x, v.y, down[j]), z(v.z, v.w, down[j]);
#pragma unroll
                for (int k = 0; k < kParts; ++k) vs[k][r][j] = x.part[k], vs[k][r][2 + j] = z.part[k];
            }
    }
    const T16* b = reinterpret_cast<const T16*>(p.b) + (int64_t)u.adapter * p.N * p.rank;
    float* out = reinterpret_cast<float*>(smem) + warp * 16 * M::kOutPitch;
    const int blocks = (p.N + 63) / 64, token0 = u.token + 16 * m, live_tokens = min(16, u.n - 16 * m);
    const typename O::T* base = reinterpret_cast<const typename O::T*>(p.base) + (int64_t)token0 * p.ldb;
    typename O::T* y = reinterpret_cast<typename O::T*>(p.y) + (int64_t)token0 * p.ldy;
    if (live_tokens > 0) {
        for (int block = part * (kWarps / 2) + (warp >> 1); block < blocks; block += parts * (kWarps / 2)) {
            const int n0 = 64 * block;
            const bool vec = p.vec && n0 + 64 <= p.N;
            // base's tile is on its way meanwhile: kRowsAtOnce rows in pieces of 16 bytes, or two elements a row
            constexpr int kPiece = 16 / sizeof(typename O::T), kLanes = 64 / kPiece, kRowsAtOnce = 32 / kLanes, kPieces = 16 / kRowsAtOnce;
            uint32_t raw[32];
            if (vec) {
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    const int row = min(kRowsAtOnce * i + lane / kLanes, live_tokens - 1);
                    uint4 x = make_uint4(0, 0, 0, 0);
                    if (p.base) x = *reinterpret_cast<const uint4*>(base + (int64_t)row * p.ldb + n0 + kPiece * (lane % kLanes));
                    raw[4 * i] = x.x, raw[4 * i + 1] = x.y, raw[4 * i + 2] = x.z, raw[4 * i + 3] = x.w;
                }
            } else {
                const typename O::T* from = base + n0 + lane;
                const bool in[2] = {p.base && n0 + lane < p.N, p.base && n0 + lane + 32 < p.N};
#pragma unroll
                for (int row = 0; row < 16; ++row, from += p.ldb)
#pragma unroll
                    for (int c = 0; c < 2; ++c) raw[2 * row + c] = in[c] && row < live_tokens ? __float_as_uint(O::load(from + 32 * c)) : 0;
            }
            float d[8][4];
            constexpr int kAtOnce = kRT <= 2 ? 4 : 2;  // tiles of 8 columns whose rows of B are on their way together
#pragma unroll
            for (int i0 = 0; i0 < 8; i0 += kAtOnce) {
                uint2 w[kAtOnce][kRT];
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                    const int n = n0 + 8 * (i0 + i) + g;
                    const T16* from = b + (int64_t)n * p.rank + 4 * t;
#pragma unroll
                    for (int r = 0; r < kRT; ++r) w[i][r] = load8_if(from + 16 * r, n < p.N && 16 * r + 4 * t < p.rank);
                }
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                    float(&to)[4] = d[i0 + i];
#pragma unroll
                    for (int j = 0; j < 4; ++j) to[j] = 0.0f;
#pragma unroll
                    for (int r = 0; r < kRT; ++r)
#pragma unroll
                        for (int k = kParts - 1; k >= 0; --k) mma_16816<kBf16>(to, vs[k][r], w[i][r].x, w[i][r].y);
                }
            }
            // through shared memory, so that a warp reads base and writes y along the rows
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    *reinterpret_cast<float2*>(out + (8 * j + g) * M::kOutPitch + 8 * i + 2 * t) = make_float2(d[i][2 * j] * back[j], d[i][2 * j + 1] * back[j]);
            __syncwarp();
            if (vec) {
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    const int row = kRowsAtOnce * i + lane / kLanes, c = kPiece * (lane % kLanes);
                    const float4 s0 = *reinterpret_cast<const float4*>(out + row * M::kOutPitch + c);
                    uint4 x;
                    if constexpr (kF32) {
                        x = make_uint4(__float_as_uint(s0.x + __uint_as_float(raw[4 * i])), __float_as_uint(s0.y + __uint_as_float(raw[4 * i + 1])),
                                       __float_as_uint(s0.z + __uint_as_float(raw[4 * i + 2])), __float_as_uint(s0.w + __uint_as_float(raw[4 * i + 3])));
                    } else {
                        const float4 s1 = *reinterpret_cast<const float4*>(out + row * M::kOutPitch + c + 4);
                        const float2 o0 = Half<kBf16>::unpack(raw[4 * i]), o1 = Half<kBf16>::unpack(raw[4 * i + 1]);
                        const float2 o2 = Half<kBf16>::unpack(raw[4 * i + 2]), o3 = Half<kBf16>::unpack(raw[4 * i + 3]);
                        x = make_uint4(Half<kBf16>::pack(s0.x + o0.x, s0.y + o0.y), Half<kBf16>::pack(s0.z + o1.x, s0.w + o1.y),
                                       Half<kBf16>::pack(s1.x + o2.x, s1.y + o2.y), Half<kBf16>::pack(s1.z + o3.x, s1.w + o3.y));
                    }
                    if (row < live_tokens) *reinterpret_cast<uint4*>(y + (int64_t)row * p.ldy + n0 + c) = x;
                }
            } else {
                typename O::T* to = y + n0 + lane;
                const bool in[2] = {n0 + lane < p.N, n0 + lane + 32 < p.N};
#pragma unroll
                for (int row = 0; row < 16; ++row, to += p.ldy)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        if (in[c] && row < live_tokens) O::store(to + 32 * c, out[row * M::kOutPitch + lane + 32 * c] + __uint_as_float(raw[2 * row + c]));
            }
            __syncwarp();
        }
    }
    cluster.barrier_wait();  // no block leaves while its sums are read
}

template <class Kernel>
cudaError_t launch(Kernel kernel, const AdapterParams& p, int64_t units, int parts, int smem, cudaStream_t st) {
    cudaLaunchAttribute attr[2] = {early_launch_attribute(), cluster_attribute(1)};
    attr[1].val.clusterDim.x = parts, attr[1].val.clusterDim.y = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * parts));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}
// Blocks of a cluster: the most, a power of two, with which all units that may not be empty are resident at once and every warp has a step of k.
// Fewer large clusters fit than the SMs have room for (17 units of rank 64 take 13.5 us in clusters of 16 and 8.8 in clusters of 8), so
// the runtime is asked, once per device and size; `fit`: what it said, plus 1.
template <class Kernel>
int cluster_of(Kernel kernel, const AdapterParams& p, int64_t units, int most, int smem, std::atomic<int> (&fit)[5]) {
    const int64_t live = std::min(units, (int64_t)p.T), steps = (p.K + 31) / 32;
    for (int log2 = most == 16 ? 4 : 3, parts = most; log2 > 0; --log2, parts /= 2) {
        if (steps < (int64_t)kWarps * parts) continue;
        int n = fit[log2].load(std::memory_order_relaxed) - 1;
        if (n < 0) {
            cudaLaunchAttribute attr = cluster_attribute(1);
            attr.val.clusterDim.x = parts, attr.val.clusterDim.y = 1;
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(parts), cfg.blockDim = dim3(kThreads), cfg.dynamicSmemBytes = smem, cfg.attrs = &attr, cfg.numAttrs = 1;
            // clusters of 16 not every GPU can have
            if ((parts > 8 && cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) ||
                cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
                cudaGetLastError();
                n = 0;
            }
            fit[log2].store(n + 1, std::memory_order_relaxed);
        }
        if (live <= n) return parts;
    }
    return 1;
}
template <bool kBf16, bool kF32, int kRT>
cudaError_t launch_rank(const AdapterParams& p, bool few, int64_t units, int device, cudaStream_t st) {
    static std::atomic<int> fit_few[64][5], fit_many[64][5];
    static std::atomic<uint64_t> done{0};
    if (few) {
        const auto kernel = adapters_few_kernel<kBf16, kF32, kRT>;
        return launch(kernel, p, units, cluster_of(kernel, p, units, kMostCluster, 0, fit_few[device & 63]), 0, st);
    }
    using M = Many<2 * kRT>;
    const auto kernel = adapters_many_kernel<kBf16, kF32, 2 * kRT>;
    const cudaError_t e = allow_smem(kernel, M::kSmemBytes, device, done);
    if (e != cudaSuccess) return e;
    return launch(kernel, p, units, cluster_of(kernel, p, units, 8, M::kSmemBytes, fit_many[device & 63]), M::kSmemBytes, st);
}
template <bool kBf16, bool kF32>
cudaError_t launch_type(const AdapterParams& p, bool few, int64_t units, int device, cudaStream_t st) {
    return p.rank <= 16   ? launch_rank<kBf16, kF32, 1>(p, few, units, device, st)
           : p.rank <= 32 ? launch_rank<kBf16, kF32, 2>(p, few, units, device, st)
           : p.rank <= 64 ? launch_rank<kBf16, kF32, 4>(p, few, units, device, st)
                          : launch_rank<kBf16, kF32, 8>(p, few, units, device, st);
}

}  // namespace
}  // namespace awe

using namespace awe;

extern "C" awe_status_t awe_linear_adapters(awe_handle_t h, const awe_adapters* L, const void* x_dev, int64_t T, int64_t ldx,
                                            const int32_t* q_start_dev, const int32_t* adapter_dev, int64_t B, const void* base_dev,
                                            int64_t ldb, void* y_dev, awe_float_t y_type, int64_t ldy, void* stream) {
    if (!h || !L || !L->a_dev || !L->b_dev || L->n_adapters <= 0 || L->rank <= 0 || L->N <= 0 || L->K <= 0 || T < 0 || B < 0) return AWE_ERR_INVALID_ARG;
    if (L->type < AWE_F16 || L->type > AWE_F32 || (int)y_type < AWE_F16 || (int)y_type > AWE_F32) return AWE_ERR_INVALID_ARG;
    if (!is_half_type(L->type) || ((int)y_type != L->type && y_type != AWE_F32) || L->rank > 128 || L->rank % 8 || L->K % 8) return AWE_ERR_UNSUPPORTED;
    // columns are counted in 32 bits, and loops look up to 32,768 of them beyond the last (copy_base: 16 blocks' threads, eight elements each)
    if (L->N > INT32_MAX - 65536 || L->K > INT32_MAX - 65536 || T > INT32_MAX - 64 || B > AWE_KV_MAX_REQUESTS) return AWE_ERR_UNSUPPORTED;
    if (T == 0 || B == 0) return AWE_OK;
    if (!x_dev || !y_dev || !q_start_dev || !adapter_dev || (T > 1 && (ldx < L->K || ldy < L->N || (base_dev && ldb < L->N))) ||
        (base_dev == y_dev && T > 1 && ldb != ldy))
        return AWE_ERR_INVALID_ARG;
    const int out = y_type == AWE_F32 ? 4 : 2;
    if ((uintptr_t)L->a_dev % 16 || (uintptr_t)L->b_dev % 16 || (uintptr_t)L->scale_dev % 4 || (uintptr_t)x_dev % 16 || (T > 1 && ldx % 8) ||
        (uintptr_t)base_dev % out || (uintptr_t)y_dev % out || (uintptr_t)q_start_dev % 4 || (uintptr_t)adapter_dev % 4)
        return AWE_ERR_ALIGNMENT;
    AdapterParams p = {};
    p.a = L->a_dev, p.b = L->b_dev, p.x = x_dev, p.base = base_dev, p.y = y_dev, p.scale = L->scale_dev;
    p.q_start = q_start_dev, p.adapter = adapter_dev, p.ldx = ldx, p.ldb = ldb, p.ldy = ldy, p.n_adapters = L->n_adapters;
    p.T = (int)T, p.B = (int)B, p.N = (int)L->N, p.K = (int)L->K, p.rank = (int)L->rank;
    p.vec = (uintptr_t)base_dev % 16 == 0 && (uintptr_t)y_dev % 16 == 0 && (!base_dev || ldb * out % 16 == 0) && ldy * out % 16 == 0;
    // Units of 8 tokens while they leave room for two blocks' clusters or hold no more than two tokens; then units of 32, which read an
    // adapter less often.  4,096 x 4,096, rank 16, units of 8 and of 32 tokens, us: one request of 8 tokens 3.9 and 6.3, of 64 5.0 and 7.4, of
    // 512 (65 units of 8) 8.0 and 9.8, of 1,024 (129) 17.1 and 10.9; 16 requests of 16 tokens 7.3 and 8.4, 32 of 16 (96) 10.1 and 9.6,
    // 64 of 8 (128) 17.4 and 15.3, 128 of 4 16.2 and 15.5; 128 of 1 11.3 and 12.3, 256 of 1 19.3 and 20.7.
    const bool few = 2 * (T / kFew + B) <= h->sm_count || T <= 2 * B;
    const int64_t units = T / (few ? kFew : kMany) + B;
    if (units > INT32_MAX / kMostCluster) return AWE_ERR_UNSUPPORTED;
    cudaStream_t st = (cudaStream_t)stream;
    const bool f32 = y_type == AWE_F32;
    const cudaError_t e = L->type == AWE_BF16 ? (f32 ? launch_type<true, true>(p, few, units, h->device, st) : launch_type<true, false>(p, few, units, h->device, st))
                                              : (f32 ? launch_type<false, true>(p, few, units, h->device, st) : launch_type<false, false>(p, few, units, h->device, st));
    if (e != cudaSuccess) return AWE_ERR_CUDA;
    h->launches += 1;
    return AWE_OK;
}
