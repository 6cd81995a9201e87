// Linear layer with 4-bit weights and group scales (awe_linear_w4).
//
//   y(m, n) = sum over groups G of scale(n, G) * sum over k in G of x(m, k) (code(n, k) - zero(n, G))
//
// A code less its zero point is an integer of 5 bits, exact in FP16 and BF16, so the inner sum runs on the 16-bit
// matrix instruction with FP32 sums and the scale is applied once per group in FP32.  Rows of the instruction are 16
// rows of the weight, its columns 8 rows of x.  With few rows of x the weight's bytes (K / 2 per row, read once) are
// the bound.
//
// A block takes 64 rows of the weight and a part of K; up to 8 blocks along K form a cluster and add their sums
// through each other's shared memory in a fixed order.  A warp's 16 rows pass through a ring of cp.async stages of
// 256 k.  Thread (g, t) of a warp reads 8 consecutive k of its rows as one word; which k takes which place in the
// instruction does not matter as long as x is placed alike, so codes are used in the order in which they unpack:
// (0,4), (1,5), (2,6), (3,7).
#include <cooperative_groups.h>

#include <algorithm>

#include "awe_internal.h"
#include "serve_common.cuh"

namespace awe {
namespace {

using namespace serve;

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kRowsN = 16 * kWarps;      // rows of the weight per block
constexpr int kStageK = 256;             // k per stage
constexpr int kPitch = kStageK / 2 + 16; // bytes per row and stage: the last 16 hold what an unaligned row spills over, and
                                         // make 8 rows x 4 words hit all banks
constexpr int kGroupsMax = kStageK / 32;
constexpr int kStages = 4;
constexpr int kMaxCluster = 8;
constexpr int kSlabK = 2048;             // k of x held at a time

struct LinearParams {
    const uint8_t* codes;
    const void* scale;
    const int8_t* zero;
    const void* x;
    void* y;
    int64_t row_bytes, ldx, ldy, codes_bytes;
    int M, N, K, group_log2, groups, k_per_block;
    int scale_bf16, y_f32, x_vec;
};

template <int kMT>
struct Config {
    static constexpr int kRowsM = 8 * kMT;
    static constexpr int kSlabPitch = kSlabK * 2 + 64;  // bytes
    static constexpr int kStageBytes = kRowsN * kPitch;
    static constexpr int kScaleBytes = kRowsN * (kGroupsMax + 1) * 8;  // (scale, zero constant) of a stage
    static constexpr int kXBytes = kRowsM * kSlabPitch;
    static constexpr int kRingBytes = kStages * (kStageBytes + kScaleBytes);
    static constexpr int kSmemBytes = kXBytes + kRingBytes;
    static constexpr int kSumBytes = kRowsM * (kRowsN + 4) * 4;  // in the place of x
};

// Nibbles i and i + 4 of a word as a pair of 16-bit floats, less `offset` = pattern bias + 8 + zero.
//   FP16: 0x6400 | u = 1024 + u, and with the nibble four bits up 1024 + 16 u = 16 (64 + u)
//   BF16: 0x4300 | u = 128 + u
// The code's sign bit is flipped by the same logic operation (u = code + 8).
template <bool kBf16>
__device__ __forceinline__ void unpack_word(uint32_t w, uint32_t offset, uint32_t offset16, uint32_t (&f)[4]) {
    if constexpr (kBf16) {
        const __nv_bfloat162 off = *reinterpret_cast<const __nv_bfloat162*>(&offset);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t v = ((w >> (4 * i)) & 0x000F000Fu) ^ 0x43084308u;
            const __nv_bfloat162 h = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), off);
            f[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
    } else {
        const __half2 off = *reinterpret_cast<const __half2*>(&offset), off16 = *reinterpret_cast<const __half2*>(&offset16);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t lo = (w & 0x000F000Fu) ^ 0x64086408u, hi = (w & 0x00F000F0u) ^ 0x64806480u;
            const __half2 a = __hsub2(*reinterpret_cast<const __half2*>(&lo), off);
            const __half2 b = __hfma2(*reinterpret_cast<const __half2*>(&hi), __float2half2_rn(0.0625f), off16);
            f[2 * i] = *reinterpret_cast<const uint32_t*>(&a);
            f[2 * i + 1] = *reinterpret_cast<const uint32_t*>(&b);
            w >>= 8;
        }
    }
}

template <int kMT, bool kBf16, bool kAligned>
__global__ void __launch_bounds__(kThreads) linear_w4_kernel(const LinearParams p) {
    namespace cg = cooperative_groups;
    using C = Config<kMT>;
    using T16 = typename Half<kBf16>::type;
    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int n0 = blockIdx.x * kRowsN, m0 = blockIdx.z * C::kRowsM, k0 = blockIdx.y * p.k_per_block;
    const int k1 = min(p.K, k0 + p.k_per_block), n_stages = k1 > k0 ? (k1 - k0 + kStageK - 1) / kStageK : 0;
    const int rows_m = min(C::kRowsM, p.M - m0);
    const uint32_t smem_at = (uint32_t)__cvta_generic_to_shared(smem), ring = smem_at + C::kXBytes;
    uint8_t* scales = smem + C::kXBytes + kStages * C::kStageBytes;

    // 16-byte pieces of a stage: 8 per row, and a ninth where rows start between 16-byte boundaries
    constexpr int kPieces = kAligned ? 8 : 9;
    auto fetch = [&](int i) {
        if (i < n_stages) {
            const int kb = (k0 + i * kStageK) >> 1, k_bytes = (min(k1 - k0 - i * kStageK, kStageK) + 1) >> 1;
            const uint32_t stage = ring + (i % kStages) * C::kStageBytes;
            for (int j = tid; j < kRowsN * kPieces; j += kThreads) {
                const int row = j / kPieces, c = j % kPieces;
                const bool live = n0 + row < p.N;
                const uint8_t* src = p.codes + (int64_t)(n0 + (live ? row : 0)) * p.row_bytes + kb;
                const int shift = kAligned ? 0 : (int)((uintptr_t)src & 15);
                const uint8_t* piece = src - shift + 16 * c;
                const int bytes = live ? min(16, max(0, k_bytes + shift - 16 * c)) : 0;
                const uint32_t dst = stage + row * kPitch + 16 * c;
                if (kAligned || piece >= p.codes) cp_async16(dst, bytes ? piece : p.codes - ((uintptr_t)p.codes & 15), bytes);
                else  // the bytes in front of the matrix are not ours to read
                    for (int e = 0; e < 16; ++e)
                        asm volatile("st.shared.u8 [%0], %1;" ::"r"(dst + e), "r"((uint32_t)(piece + e >= p.codes && e < bytes ? piece[e] : 0)) : "memory");
            }
        }
        cp_async_commit();
    };
    // scale and zero constants of a stage: element (row, group of the stage)
    const int per_stage = p.group_log2 >= 8 ? 1 : kStageK >> p.group_log2;
    auto put_scales = [&](int i) {
        if (i >= n_stages) return;
        const int first = (k0 + i * kStageK) >> p.group_log2;
        for (int j = tid; j < kRowsN * per_stage; j += kThreads) {
            const int row = j / per_stage, gi = j % per_stage;
            float s = 0.0f;
            int z = 0;
            if (n0 + row < p.N && first + gi < p.groups) {
                const int64_t at = (int64_t)(n0 + row) * p.groups + first + gi;
                s = p.scale_bf16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p.scale)[at]) : __half2float(reinterpret_cast<const __half*>(p.scale)[at]);
                if (p.zero) z = (int)((uint32_t)(uint8_t)p.zero[at] << 28) >> 28;
            }
            const float bias = kBf16 ? 136.0f : 1032.0f;
            const uint32_t off = kBf16 ? Half<true>::pack(bias + z, bias + z) : Half<false>::pack(bias + z, 0.0f - (72.0f + z));
            *reinterpret_cast<uint2*>(scales + (i % kStages) * C::kScaleBytes + (row * (kGroupsMax + 1) + gi) * 8) = make_uint2(__float_as_uint(s), off);
        }
    };
    // x for [k0 + at, + kSlabK), zeros behind the block's part of K and below the last row
    auto load_x = [&](int at) {
        const int n_k = min(kSlabK, k1 - k0 - at), n_round = (n_k + kStageK - 1) / kStageK * kStageK;
        for (int j = tid; j < rows_m * (n_round / 8); j += kThreads) {
            const int row = j / (n_round / 8), k = j % (n_round / 8) * 8;
            const T16* src = reinterpret_cast<const T16*>(p.x) + (int64_t)(m0 + row) * p.ldx + k0 + at + k;
            uint32_t w[4] = {0, 0, 0, 0};
            if (p.x_vec && k + 8 <= n_k) {
                const uint4 v = __ldg(reinterpret_cast<const uint4*>(src));
                w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (k + e < n_k) w[e >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(src)[e] << (16 * (e & 1));
            }
            // pairs (0,4), (1,5), (2,6), (3,7)
            *reinterpret_cast<uint4*>(smem + row * C::kSlabPitch + k * 2) =
                make_uint4(__byte_perm(w[0], w[2], 0x5410), __byte_perm(w[0], w[2], 0x7632), __byte_perm(w[1], w[3], 0x5410),
                           __byte_perm(w[1], w[3], 0x7632));
        }
    };

    float total[kMT][4];
#pragma unroll
    for (int mt = 0; mt < kMT; ++mt) total[mt][0] = total[mt][1] = total[mt][2] = total[mt][3] = 0.0f;

#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch(i);
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) put_scales(i);
    // where a row starts inside its first 16 bytes
    const int row_a = 16 * warp + g, row_b = row_a + 8;
    auto shift_of = [&](int row) { return kAligned ? 0 : (int)((uintptr_t)(p.codes + (int64_t)(n0 + min(row, p.N - 1 - n0)) * p.row_bytes + (k0 >> 1)) & 15); };
    const int shift_a = shift_of(row_a), shift_b = shift_of(row_b);
    const int steps_per_scale = p.group_log2 >= 8 ? 8 : 1 << (p.group_log2 - 5);

    for (int i = 0; i < n_stages; ++i) {
        if (i % (kSlabK / kStageK) == 0) {
            __syncthreads();
            load_x(i * kStageK);
        }
        cp_async_wait<kStages - 2>();
        __syncthreads();
        fetch(i + kStages - 1);
        put_scales(i + kStages - 1);
        const uint32_t stage = ring + (i % kStages) * C::kStageBytes;
        const uint32_t at_a = stage + row_a * kPitch + (shift_a & ~3) + 4 * t, at_b = stage + row_b * kPitch + (shift_b & ~3) + 4 * t;
        const uint32_t x_at = smem_at + g * C::kSlabPitch + (i % (kSlabK / kStageK)) * kStageK * 2 + 16 * t;
        const uint8_t* sc = scales + (i % kStages) * C::kScaleBytes;
        for (int gi = 0; gi < per_stage; ++gi) {
            const uint2 sa = *reinterpret_cast<const uint2*>(sc + (row_a * (kGroupsMax + 1) + gi) * 8);
            const uint2 sb = *reinterpret_cast<const uint2*>(sc + (row_b * (kGroupsMax + 1) + gi) * 8);
            const uint32_t off_a = __byte_perm(sa.y, 0, 0x1010), off_b = __byte_perm(sb.y, 0, 0x1010);
            const uint32_t off16_a = __byte_perm(sa.y, 0, 0x3232), off16_b = __byte_perm(sb.y, 0, 0x3232);
            float acc[kMT][4];
#pragma unroll
            for (int mt = 0; mt < kMT; ++mt) acc[mt][0] = acc[mt][1] = acc[mt][2] = acc[mt][3] = 0.0f;
#pragma unroll 2
            for (int j = 0; j < steps_per_scale; ++j) {
                const int c = gi * steps_per_scale + j;  // 32 k
                uint32_t wa = lds32(at_a + 16 * c), wb = lds32(at_b + 16 * c);
                if constexpr (!kAligned) {
                    wa = __funnelshift_r(wa, lds32(at_a + 16 * c + 4), 8 * (shift_a & 3));
                    wb = __funnelshift_r(wb, lds32(at_b + 16 * c + 4), 8 * (shift_b & 3));
                }
                uint32_t fa[4], fb[4];
                unpack_word<kBf16>(wa, off_a, off16_a, fa);
                unpack_word<kBf16>(wb, off_b, off16_b, fb);
                const uint32_t a0[4] = {fa[0], fb[0], fa[1], fb[1]}, a1[4] = {fa[2], fb[2], fa[3], fb[3]};
#pragma unroll
                for (int mt = 0; mt < kMT; ++mt) {
                    uint4 x = make_uint4(0, 0, 0, 0);
                    if (8 * mt + g < rows_m) x = lds128(x_at + mt * 8 * C::kSlabPitch + 64 * c);
                    mma_16816<kBf16>(acc[mt], a0, x.x, x.y);
                    mma_16816<kBf16>(acc[mt], a1, x.z, x.w);
                }
            }
            const float s_a = __uint_as_float(sa.x), s_b = __uint_as_float(sb.x);
#pragma unroll
            for (int mt = 0; mt < kMT; ++mt) {
                total[mt][0] = fmaf(acc[mt][0], s_a, total[mt][0]);
                total[mt][1] = fmaf(acc[mt][1], s_a, total[mt][1]);
                total[mt][2] = fmaf(acc[mt][2], s_b, total[mt][2]);
                total[mt][3] = fmaf(acc[mt][3], s_b, total[mt][3]);
            }
        }
    }
    cp_async_wait<0>();
    __syncthreads();

    // ---- sums to shared memory as (row of x, row of the weight), then the cluster's blocks add them
    float* sums = reinterpret_cast<float*>(smem);
    constexpr int kSumPitch = kRowsN + 4;
#pragma unroll
    for (int mt = 0; mt < kMT; ++mt)
#pragma unroll
        for (int j = 0; j < 4; ++j) sums[(8 * mt + 2 * t + (j & 1)) * kSumPitch + (j >> 1 ? row_b : row_a)] = total[mt][j];
    cg::cluster_group cluster = cg::this_cluster();
    const int parts = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    if (parts > 1) cluster.sync();
    else __syncthreads();
    const float* from[kMaxCluster];
#pragma unroll
    for (int r = 0; r < kMaxCluster; ++r) from[r] = r < parts ? cluster.map_shared_rank(sums, r) : sums;
    for (int j = rank * kThreads + tid; j < rows_m * kRowsN; j += parts * kThreads) {
        const int m = j / kRowsN, n = j % kRowsN;
        if (n0 + n >= p.N) continue;
        float v = 0.0f;
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r)
            if (r < parts) v += from[r][m * kSumPitch + n];
        const int64_t at = (int64_t)(m0 + m) * p.ldy + n0 + n;
        if (p.y_f32) reinterpret_cast<float*>(p.y)[at] = v;
        else reinterpret_cast<T16*>(p.y)[at] = Half<kBf16>::from_float(v);
    }
    if (parts > 1) cluster.sync();  // no block leaves while its sums are read
}

template <int kMT, bool kBf16, bool kAligned>
cudaError_t launch(const LinearParams& p, int parts, cudaStream_t st) {
    using C = Config<kMT>;
    static_assert(C::kSumBytes <= C::kXBytes, "the sums take the place of x");
    cudaError_t e = cudaFuncSetAttribute(linear_w4_kernel<kMT, kBf16, kAligned>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((p.N + kRowsN - 1) / kRowsN, parts, (p.M + C::kRowsM - 1) / C::kRowsM);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = C::kSmemBytes;
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 1;
    attr.val.clusterDim.y = parts;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, linear_w4_kernel<kMT, kBf16, kAligned>, p);
}
template <int kMT>
cudaError_t launch(const LinearParams& p, bool bf16, bool aligned, int parts, cudaStream_t st) {
    if (bf16) return aligned ? launch<kMT, true, true>(p, parts, st) : launch<kMT, true, false>(p, parts, st);
    return aligned ? launch<kMT, false, true>(p, parts, st) : launch<kMT, false, false>(p, parts, st);
}

}  // namespace
}  // namespace awe

using namespace awe;

extern "C" awe_status_t awe_linear_w4(awe_handle_t h, const awe_w4_matrix* W, const void* x_dev, awe_float_t x_type,
                                      int64_t M, int64_t ldx, void* y_dev, awe_float_t y_type, int64_t ldy, void* stream) {
    if (!h || !W || !W->codes_dev || !W->scale_dev || W->N <= 0 || W->K <= 0 || M < 0 || W->ld < W->K || (W->ld & 1))
        return AWE_ERR_INVALID_ARG;
    if (W->group < 32 || (W->group & (W->group - 1))) return AWE_ERR_UNSUPPORTED;
    if ((int)x_type < AWE_F16 || (int)x_type > AWE_F32 || (int)y_type < AWE_F16 || (int)y_type > AWE_F32 ||
        W->scale_type < AWE_F16 || W->scale_type > AWE_F32)
        return AWE_ERR_INVALID_ARG;
    if (!is_half_type(x_type) || !is_half_type(W->scale_type) || (y_type != x_type && y_type != AWE_F32)) return AWE_ERR_UNSUPPORTED;
    if (W->N > INT32_MAX - 256 || W->K > INT32_MAX - 4096 || M > 65535 * 8) return AWE_ERR_UNSUPPORTED;
    if (M == 0) return AWE_OK;
    if (!x_dev || !y_dev || (M > 1 && (ldx < W->K || ldy < W->N))) return AWE_ERR_INVALID_ARG;
    if ((uintptr_t)x_dev % 2 || (uintptr_t)W->scale_dev % 2 || (uintptr_t)y_dev % (y_type == AWE_F32 ? 4 : 2)) return AWE_ERR_ALIGNMENT;
    LinearParams p = {};
    p.codes = (const uint8_t*)W->codes_dev, p.scale = W->scale_dev, p.zero = W->zero_dev, p.x = x_dev, p.y = y_dev;
    p.row_bytes = W->ld / 2, p.ldx = ldx, p.ldy = ldy;
    p.M = (int)M, p.N = (int)W->N, p.K = (int)W->K;
    while ((int64_t)1 << p.group_log2 < W->group && p.group_log2 < 31) ++p.group_log2;
    p.groups = (int)((W->K + W->group - 1) / W->group);
    p.scale_bf16 = W->scale_type == AWE_BF16, p.y_f32 = y_type == AWE_F32;
    p.x_vec = (uintptr_t)x_dev % 16 == 0 && (ldx % 8 == 0 || M == 1);
    const bool aligned = (uintptr_t)W->codes_dev % 16 == 0 && W->ld % 32 == 0;
    const int tiles_m = M <= 8 ? 1 : (M <= 16 ? 2 : 4);
    // Parts of K: enough blocks for about three per SM, each with two stages at least.
    const int64_t tiles = (p.N + kRowsN - 1) / kRowsN * ((M + 8 * tiles_m - 1) / (8 * tiles_m));
    int parts = 1;
    while (parts < kMaxCluster && tiles * parts < 3 * h->sm_count && p.K > 2 * parts * 2 * kStageK) parts *= 2;
    p.k_per_block = (int)round_up((p.K + parts - 1) / parts, kStageK);
    cudaStream_t st = (cudaStream_t)stream;
    const bool bf16 = x_type == AWE_BF16;
    const cudaError_t e = tiles_m == 1   ? launch<1>(p, bf16, aligned, parts, st)
                          : tiles_m == 2 ? launch<2>(p, bf16, aligned, parts, st)
                                         : launch<4>(p, bf16, aligned, parts, st);
    if (e != cudaSuccess) return AWE_ERR_CUDA;
    h->launches += 1;
    return AWE_OK;
}
