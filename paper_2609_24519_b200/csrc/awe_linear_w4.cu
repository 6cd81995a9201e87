// Linear layer with 4-bit weights and group scales (awe_linear_w4).
//
//   y(m, n) = sum over groups G of scale(n, G) * sum over k in G of x(m, k) (code(n, k) - zero(n, G))
//
// A code less its zero point is an integer of 5 bits, exact in FP16 and BF16, so the inner sum runs on the 16-bit
// matrix instruction with FP32 sums and the scale is applied once per group in FP32.  Rows of the instruction are 16
// rows of the weight, its columns 8 rows of x.  With few rows of x the weight's bytes (K / 2 per row, read once) are
// the bound.
//
// A warp takes 16 rows of the weight and a part of K.  One or two rows of x: a block of eight warps cuts K into 1, 2, 4 or 8
// slices and adds them at its end (4,096 x 4,096 for one row: 8.2 -> 5.2 us a call, since a launch of clusters takes longer
// than the product).  Otherwise a block is four warps with 64 rows that share x, and up to 8 blocks along K form a cluster
// and add their sums through each other's shared memory.  All sums are added in a fixed order.  A warp has a ring of its own:
// a stage is 256 k of the codes (cp.async, 16 bytes a piece), and the stage that begins a slab (512 to 4,096 k) brings the
// slab's scales and zero points along, so that a warp waits for nobody but itself within a slab.  Thread (g, t) of a warp reads
// 8 consecutive k of its rows as one word; which k takes which place in the instruction does not matter as long as x
// is placed alike, so codes are used in the order in which they unpack: (0,4), (1,5), (2,6), (3,7).
#include <cooperative_groups.h>

#include <algorithm>

#include "linear_w4.cuh"

namespace awe {
namespace {

using namespace serve;

constexpr int kSliceWarps = 8, kShareWarps = 4;  // warps of a block that cuts K, or shares x
constexpr int kWarpRows = 16;
constexpr int kStageK = 256;                // k per stage
constexpr int kPitch = kStageK / 2 + 16;    // bytes per row and stage: the last 16 hold what an unaligned row spills over, and
                                            // make 8 rows x 4 words hit all banks
constexpr int kStageBytes = kWarpRows * kPitch;
constexpr int kStages = 3;
constexpr int kZeroBytes = kStageK * 2 + 128;  // read in the place of rows of x that do not exist
constexpr int kMaxCluster = 8;
constexpr int kSlabKMost = 4096;   // k whose x, scales and zero points are held at a time, at most
constexpr int kXMost = 17 * 1024;  // bytes of x of the slabs of a block, about

struct LinearParams {
    const uint8_t* codes;
    const uint8_t* scale;
    const uint8_t* zero;
    const void* x;
    void* y;
    int64_t row_bytes, ldx, ldy;
    int M, N, K, group_log2, groups, k_per_block, k_per_slice, slice_log2, slab_count;
    int scale_bf16, y_f32, x_vec;
    int scale_pitch, zero_pitch;  // bytes of a row's scales and zero points of a slab, with room for what an unaligned row spills over
    int ring_at, slab_at;         // byte offsets in shared memory: x first
    int slabs;                    // 2 where a block has more than one
    int slab_stages;              // a power of two
    int device;
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
            const uint32_t v = and_xor(w >> (4 * i), 0x000F000Fu, 0x43084308u);
            const __nv_bfloat162 h = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), off);
            f[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
    } else {
        const __half2 off = *reinterpret_cast<const __half2*>(&offset), off16 = *reinterpret_cast<const __half2*>(&offset16);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t lo = and_xor(w, 0x000F000Fu, 0x64086408u), hi = and_xor(w, 0x00F000F0u, 0x64806480u);
            const __half2 a = __hsub2(*reinterpret_cast<const __half2*>(&lo), off);
            const __half2 b = __hfma2(*reinterpret_cast<const __half2*>(&hi), __float2half2_rn(0.0625f), off16);
            f[2 * i] = *reinterpret_cast<const uint32_t*>(&a);
            f[2 * i + 1] = *reinterpret_cast<const uint32_t*>(&b);
            w >>= 8;
        }
    }
}

template <int kWarps, int kMT, int kGroupSteps, bool kBf16, bool kAligned>
__global__ void __launch_bounds__(32 * kWarps) linear_w4_kernel(const LinearParams p) {
    constexpr int kThreads = 32 * kWarps;
    namespace cg = cooperative_groups;
    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    grid_wait();
    // this warp: 16 rows, a slice of k
    const int slice_log2 = kWarps == kShareWarps ? 0 : p.slice_log2;
    const int row_warps = kWarps >> slice_log2, slice = warp / row_warps, row_warp = warp % row_warps, block_rows = kWarpRows * row_warps;
    const int n0 = blockIdx.x * block_rows, m0 = blockIdx.z * 8 * kMT, k0 = blockIdx.y * p.k_per_block + slice * p.k_per_slice;
    const int k1 = min(p.K, min(k0 + p.k_per_slice, (int)(blockIdx.y + 1) * p.k_per_block)), n_stages = k1 > k0 ? (k1 - k0 + kStageK - 1) / kStageK : 0;
    const int rows_m = min(8 * kMT, p.M - m0), slab_k = p.slab_stages * kStageK, x_pitch = slab_k * 2 + 64;
    // Rows of the weight below the last one are computed from the last one and not written.
    const int n_warp = n0 + row_warp * kWarpRows;
    uint8_t* x_slab = smem + slice * rows_m * x_pitch;
    auto row_of = [&](int row) { return (int64_t)min(n_warp + row, p.N - 1); };
    const uint32_t smem_at = (uint32_t)__cvta_generic_to_shared(smem), ring = smem_at + p.ring_at + warp * kStages * kStageBytes;
    const int slab_bytes = kWarpRows * (p.scale_pitch + p.zero_pitch);
    const uint32_t slabs = smem_at + p.slab_at + warp * p.slabs * slab_bytes;
    auto slab_of = [&](int i) { return slabs + (p.slabs == 2 && (i & p.slab_stages) ? slab_bytes : 0); };

    // aligned rows: this lane copies piece lane % 8 of the rows lane / 8 + 4 j
    const uint8_t* codes[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) codes[j] = p.codes + row_of((lane >> 3) + 4 * j) * p.row_bytes + (k0 >> 1) + 16 * (lane & 7);
    const uint32_t codes_dst = ring + (lane >> 3) * kPitch + 16 * (lane & 7);
    auto fetch = [&](int i) {
        if (i < n_stages) {
            const int k = k0 + i * kStageK, slot = i % kStages;
            if constexpr (kAligned) {
                const int bytes = k + kStageK <= k1 ? 16 : min(16, max(0, ((k1 - k + 1) >> 1) - 16 * (lane & 7)));
#pragma unroll
                for (int j = 0; j < 4; ++j) cp_async16(codes_dst + slot * kStageBytes + 4 * j * kPitch, codes[j] + (bytes ? i * (kStageK / 2) : 0), bytes);
            } else {  // a ninth piece per row; half a warp per row
                const int k_bytes = (min(k1 - k, kStageK) + 1) >> 1, c = lane & 15;
#pragma unroll 4
                for (int row = lane >> 4; row < kWarpRows; row += 2)
                    if (c < 9) copy_piece(ring + slot * kStageBytes + row * kPitch, p.codes + row_of(row) * p.row_bytes + (k >> 1), k_bytes, c, p.codes);
            }
            if ((i & (p.slab_stages - 1)) == 0) {  // two lanes per row
                const uint32_t slab = slab_of(i);
                const int first = k >> p.group_log2, n = ((min(k1, k + slab_k) - 1) >> p.group_log2) + 1 - first, row = lane >> 1;
                const int64_t at = row_of(row) * p.groups + first;
#pragma unroll 1
                for (int c = lane & 1; 16 * c < p.scale_pitch; c += 2) copy_piece(slab + row * p.scale_pitch, p.scale + 2 * at, 2 * n, c, p.scale);
#pragma unroll 1
                for (int c = lane & 1; 16 * c < p.zero_pitch; c += 2)
                    copy_piece(slab + kWarpRows * p.scale_pitch + row * p.zero_pitch, p.zero + at, n, c, p.zero);
            }
        }
        cp_async_commit();
    };
    // x for [k0 + at, + slab_k), zeros behind the slice: the slice's warps take four pieces of 256 k in turn
    auto load_x = [&](int at) {
        const int n_k = min(slab_k, k1 - k0 - at), n_round = (n_k + kStageK - 1) / kStageK * kStageK;
        const int slab_log2 = __ffs(p.slab_stages) - 1;
        for (int j0 = 4 * row_warp; j0 < rows_m * p.slab_stages; j0 += 4 * row_warps) {
            uint4 w[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int row = (j0 + u) >> slab_log2, k = ((j0 + u) & (p.slab_stages - 1)) * kStageK + 8 * lane;
                const uint16_t* src = reinterpret_cast<const uint16_t*>(p.x) + (m0 + min(row, rows_m - 1)) * p.ldx + k0 + at;
                w[u] = load_x8(src + min(k, n_k), p.x_vec, row < rows_m ? n_k - k : 0);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int row = (j0 + u) >> slab_log2, k = ((j0 + u) & (p.slab_stages - 1)) * kStageK + 8 * lane;
                // pairs (0,4), (1,5), (2,6), (3,7)
                if (row < rows_m && k < n_round)
                    *reinterpret_cast<uint4*>(x_slab + row * x_pitch + k * 2) =
                        make_uint4(__byte_perm(w[u].x, w[u].z, 0x5410), __byte_perm(w[u].x, w[u].z, 0x7632),
                                   __byte_perm(w[u].y, w[u].w, 0x5410), __byte_perm(w[u].y, w[u].w, 0x7632));
            }
        }
    };

    float total[kMT][4];
#pragma unroll
    for (int mt = 0; mt < kMT; ++mt) total[mt][0] = total[mt][1] = total[mt][2] = total[mt][3] = 0.0f;

#pragma unroll 1
    for (int i = 0; i < kStages - 1; ++i) fetch(i);
    for (int k = 16 * tid; k < kZeroBytes; k += 16 * kThreads) *reinterpret_cast<uint4*>(smem + p.ring_at - kZeroBytes + k) = make_uint4(0, 0, 0, 0);
    uint32_t x_row[kMT], x_mask[kMT];
#pragma unroll
    for (int mt = 0; mt < kMT; ++mt) {
        const bool live = 8 * mt + g < rows_m;
        x_row[mt] = smem_at + (live ? (slice * rows_m + 8 * mt + g) * x_pitch : p.ring_at - kZeroBytes) + 16 * t;
        x_mask[mt] = live ? ~0u : 0u;
    }
    // where rows g, g + 8 of the warp start inside their first 16 bytes of codes
    const int row_a = g, row_b = g + 8;
    auto shift_of = [&](int row) { return kAligned ? 0 : (int)((uintptr_t)(p.codes + row_of(row) * p.row_bytes + (k0 >> 1)) & 15); };
    const int shift_a = shift_of(row_a), shift_b = shift_of(row_b);
    const uint32_t word_a = ring + row_a * kPitch + (shift_a & ~3) + 4 * t, word_b = ring + row_b * kPitch + (shift_b & ~3) + 4 * t;
    constexpr int kScales = kStageK / 32 / kGroupSteps;  // of a stage
    uint32_t scale_a = 0, scale_b = 0, zero_a = 0, zero_b = 0;

    for (int begin = 0; begin < p.slab_count * p.slab_stages; begin += p.slab_stages) {  // slabs: as many for every warp
        if (begin) __syncthreads();
        if (begin < n_stages) {
            load_x(begin * kStageK);
            const uint32_t slab = slab_of(begin), zeros = slab + kWarpRows * p.scale_pitch;
            const int64_t at_a = row_of(row_a) * p.groups + ((k0 + begin * kStageK) >> p.group_log2), at_b = row_of(row_b) * p.groups + ((k0 + begin * kStageK) >> p.group_log2);
            scale_a = slab + row_a * p.scale_pitch + ((uint32_t)(uintptr_t)(p.scale + 2 * at_a) & 15);
            scale_b = slab + row_b * p.scale_pitch + ((uint32_t)(uintptr_t)(p.scale + 2 * at_b) & 15);
            zero_a = zeros + row_a * p.zero_pitch + ((uint32_t)(uintptr_t)(p.zero + at_a) & 15);
            zero_b = zeros + row_b * p.zero_pitch + ((uint32_t)(uintptr_t)(p.zero + at_b) & 15);
        }
        __syncthreads();
    for (int i = begin; i < min(n_stages, begin + p.slab_stages); ++i) {
        cp_async_wait<kStages - 2>();
        __syncwarp();
        fetch(i + kStages - 1);
        const uint32_t at_a = word_a + (i % kStages) * kStageBytes, at_b = word_b + (i % kStages) * kStageBytes;
        const uint32_t x_off = (i & (p.slab_stages - 1)) * kStageK * 2;
        // first group of the stage, counted from the slab's
        const int first = ((k0 + i * kStageK) >> p.group_log2) - ((k0 + (i & ~(p.slab_stages - 1)) * kStageK) >> p.group_log2);
#pragma unroll
        for (int gi = 0; gi < kScales; ++gi) {
            uint32_t raw_a, raw_b, ua = 8, ub = 8;  // zero point + 8
            asm volatile("ld.shared.u16 %0, [%1];" : "=r"(raw_a) : "r"(scale_a + 2 * first + 2 * gi));
            asm volatile("ld.shared.u16 %0, [%1];" : "=r"(raw_b) : "r"(scale_b + 2 * first + 2 * gi));
            if (p.zero) {
                asm volatile("ld.shared.u8 %0, [%1];" : "=r"(ua) : "r"(zero_a + first + gi));
                asm volatile("ld.shared.u8 %0, [%1];" : "=r"(ub) : "r"(zero_b + first + gi));
                ua = (ua & 15) ^ 8, ub = (ub & 15) ^ 8;
            }
            // patterns of bias + 8 + zero, whose last place is 1 (1/16 for -(64 + 8 + zero))
            const uint32_t off_a = ua * 0x10001u + (kBf16 ? 0x43004300u : 0x64006400u), off_b = ub * 0x10001u + (kBf16 ? 0x43004300u : 0x64006400u);
            const uint32_t off16_a = ua * 0x100010u + 0xD400D400u, off16_b = ub * 0x100010u + 0xD400D400u;
            const float s_a = p.scale_bf16 ? __uint_as_float(raw_a << 16) : __half2float(__ushort_as_half((unsigned short)raw_a));
            const float s_b = p.scale_bf16 ? __uint_as_float(raw_b << 16) : __half2float(__ushort_as_half((unsigned short)raw_b));
            float acc[kMT][4];
#pragma unroll
            for (int j = 0; j < kGroupSteps; ++j) {
                const int c = gi * kGroupSteps + j;  // 32 k
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
                    const uint4 x = lds128(x_row[mt] + (x_off & x_mask[mt]) + 64 * c);
                    if (j == 0) mma_16816_zero<kBf16>(acc[mt], a0, x.x, x.y);
                    else mma_16816<kBf16>(acc[mt], a0, x.x, x.y);
                    mma_16816<kBf16>(acc[mt], a1, x.z, x.w);
                }
            }
#pragma unroll
            for (int mt = 0; mt < kMT; ++mt) {
                total[mt][0] = fmaf(acc[mt][0], s_a, total[mt][0]);
                total[mt][1] = fmaf(acc[mt][1], s_a, total[mt][1]);
                total[mt][2] = fmaf(acc[mt][2], s_b, total[mt][2]);
                total[mt][3] = fmaf(acc[mt][3], s_b, total[mt][3]);
            }
        }
    }
    }
    cp_async_wait<0>();
    __syncthreads();

    // ---- sums to shared memory as (slice, row of x, row of the weight); the block, then the cluster, adds them
    float* sums = reinterpret_cast<float*>(smem);
    const int pitch = block_rows + 4, slices = 1 << slice_log2;
#pragma unroll
    for (int mt = 0; mt < kMT; ++mt)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            sums[(slice * 8 * kMT + 8 * mt + 2 * t + (j & 1)) * pitch + row_warp * kWarpRows + (j >> 1 ? row_b : row_a)] = total[mt][j];
    cg::cluster_group cluster = cg::this_cluster();
    const int parts = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    if (parts > 1) cluster.sync();
    else __syncthreads();
    const float* from[kMaxCluster];
#pragma unroll
    for (int r = 0; r < kMaxCluster; ++r) from[r] = kWarps == kShareWarps && r < parts ? cluster.map_shared_rank(sums, r) : sums;
    for (int j = rank * kThreads + tid; j < rows_m * block_rows; j += parts * kThreads) {
        const int m = j / block_rows, n = j % block_rows;
        if (n0 + n >= p.N) continue;
        float v = 0.0f;
        if constexpr (kWarps == kShareWarps) {
#pragma unroll
            for (int r = 0; r < kMaxCluster; ++r)
                if (r < parts) v += from[r][m * pitch + n];
        } else {
            for (int i = 0; i < slices; ++i) v += sums[(i * 8 * kMT + m) * pitch + n];
        }
        const int64_t at = (int64_t)(m0 + m) * p.ldy + n0 + n;
        if (p.y_f32) reinterpret_cast<float*>(p.y)[at] = v;
        else reinterpret_cast<typename Half<kBf16>::type*>(p.y)[at] = Half<kBf16>::from_float(v);
    }
    if (parts > 1) cluster.sync();  // no block leaves while its sums are read
}

template <int kWarps, int kMT, int kGroupSteps, bool kBf16, bool kAligned>
cudaError_t launch(LinearParams p, int parts, cudaStream_t st) {
    constexpr int kThreads = 32 * kWarps;
    // Shared memory: x of the slices' slabs (and at the end the sums in its place), the rings, the slabs' scales and zeros.
    const int rows = std::min(p.M, 8 * kMT), slices = 1 << p.slice_log2, block_rows = kWarpRows * kWarps / slices;
    int slab_k = (kStages - 1) * kStageK;  // two slabs' worth of stages are under way at most
    while (slab_k < kSlabKMost && slab_k < p.k_per_slice && 2 * slab_k * 2 * rows * slices <= kXMost) slab_k *= 2;
    const int slab_groups = std::max(1, slab_k >> p.group_log2);
    p.slab_stages = slab_k / kStageK;
    p.slab_count = (p.k_per_slice + slab_k - 1) / slab_k;
    p.scale_pitch = (int)round_up(2 * slab_groups, 16) + 16;
    p.zero_pitch = p.zero ? (int)round_up(slab_groups, 16) + 16 : 0;
    p.slabs = p.slab_count > 1 ? 2 : 1;
    p.ring_at = (int)round_up(std::max(slices * rows * (slab_k * 2 + 64), slices * 8 * kMT * (block_rows + 4) * 4) + kZeroBytes, 128);
    p.slab_at = p.ring_at + kWarps * kStages * kStageBytes;
    const int smem = p.slab_at + kWarps * p.slabs * kWarpRows * (p.scale_pitch + p.zero_pitch);
    constexpr int kMost = 227 * 1024;
    static_assert(kMT * 8 * ((kStages - 1) * kStageK * 2 + 64) + kXMost + kWarps * 2 * kWarpRows * (kSlabKMost / 32 * 3 + 32) / (kMT > 1 ? 4 : 1) + kZeroBytes + 128 + kWarps * kStages * kStageBytes <= kMost, "shared memory of a block");
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = allow_smem(linear_w4_kernel<kWarps, kMT, kGroupSteps, kBf16, kAligned>, kMost, p.device, done);
    if (e != cudaSuccess) return e;
    const dim3 grid((p.N + block_rows - 1) / block_rows, parts, (p.M + 8 * kMT - 1) / (8 * kMT));
    if (parts == 1) return launch_early(linear_w4_kernel<kWarps, kMT, kGroupSteps, kBf16, kAligned>, grid, kThreads, smem, st, p);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr = cluster_attribute(parts);
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, linear_w4_kernel<kWarps, kMT, kGroupSteps, kBf16, kAligned>, p);
}
template <int kWarps, int kMT, int kGroupSteps>
cudaError_t launch(const LinearParams& p, bool bf16, bool aligned, int parts, cudaStream_t st) {
    if (bf16)
        return aligned ? launch<kWarps, kMT, kGroupSteps, true, true>(p, parts, st) : launch<kWarps, kMT, kGroupSteps, true, false>(p, parts, st);
    return aligned ? launch<kWarps, kMT, kGroupSteps, false, true>(p, parts, st) : launch<kWarps, kMT, kGroupSteps, false, false>(p, parts, st);
}
template <int kWarps, int kMT>
cudaError_t launch(const LinearParams& p, bool bf16, bool aligned, int parts, cudaStream_t st) {
    switch (p.group_log2) {
        case 5: return launch<kWarps, kMT, 1>(p, bf16, aligned, parts, st);
        case 6: return launch<kWarps, kMT, 2>(p, bf16, aligned, parts, st);
        case 7: return launch<kWarps, kMT, 4>(p, bf16, aligned, parts, st);
        default: return launch<kWarps, kMT, 8>(p, bf16, aligned, parts, st);
    }
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
    if (W->N > INT32_MAX - 256 || W->K > INT32_MAX - 65536 || M > 65535 * 8) return AWE_ERR_UNSUPPORTED;
    if (M == 0) return AWE_OK;
    if (!x_dev || !y_dev || (M > 1 && (ldx < W->K || ldy < W->N))) return AWE_ERR_INVALID_ARG;
    if ((uintptr_t)x_dev % 2 || (uintptr_t)W->scale_dev % 2 || (uintptr_t)y_dev % (y_type == AWE_F32 ? 4 : 2)) return AWE_ERR_ALIGNMENT;
    LinearParams p = {};
    p.codes = (const uint8_t*)W->codes_dev, p.scale = (const uint8_t*)W->scale_dev, p.zero = (const uint8_t*)W->zero_dev, p.x = x_dev, p.y = y_dev;
    p.row_bytes = W->ld / 2, p.ldx = ldx, p.ldy = ldy, p.device = h->device;
    p.M = (int)M, p.N = (int)W->N, p.K = (int)W->K;
    while ((int64_t)1 << p.group_log2 < W->group && p.group_log2 < 31) ++p.group_log2;
    p.groups = (int)((W->K + W->group - 1) / W->group);
    p.scale_bf16 = W->scale_type == AWE_BF16, p.y_f32 = y_type == AWE_F32;
    p.x_vec = (uintptr_t)x_dev % 16 == 0 && (ldx % 8 == 0 || M == 1);
    const bool aligned = (uintptr_t)W->codes_dev % 16 == 0 && W->ld % 32 == 0;
    cudaStream_t st = (cudaStream_t)stream;
    // tcgen05 pays from more rows of x than two column blocks of the small instruction on, where the product is worth its setting up.
    // Times of the small kernel / tcgen05 in us, groups of 128: M = 16, 4,096 x 4,096 (N x K): 8.2 / 10.6; 16,384 x 8,192: 39 / 40.
    // M = 17, 2,048 x 8,192 (2.9e8): 12.9 / 13.5; 6,000 x 4,096 (4.2e8): 21.5 / 15.0.  M = 128, 1,024 x 2,560 (3.4e8): 10.4 / 10.6;
    // 1,024 x 4,064 (5.3e8): 14.5 / 12.5.  M = 1,024, 1,024 x 256 (2.7e8): 15.2 / 16.2; 1,024 x 1,024 (1.1e9): 28 / 14; 1,024 x 8,192:
    // 171 / 38.  Over 1,200 sizes, aligned and not, the rule is 0.7 % above the better of the two, at the worst 1.4 times.
    if (M > 16 && (double)M * W->N * W->K >= 4.5e8)
        return linear_w4_tc(h, *W, x_dev, x_type == AWE_BF16, M, ldx, y_dev, y_type == AWE_F32, ldy, st);
    const int tiles_m = M <= 8 ? 1 : (M <= 16 ? 2 : 4);
    // K is split so that about 16 warps per SM have work (what is resident at once), with two stages each at least.
    const int64_t warps = (p.N + kWarpRows - 1) / kWarpRows * ((M + 8 * tiles_m - 1) / (8 * tiles_m));
    const int split = (int)std::max<int64_t>(1, std::min<int64_t>({kSliceWarps * kMaxCluster, 16 * h->sm_count / warps, p.K / (2 * kStageK)}));
    const bool bf16 = x_type == AWE_BF16, sliced = M <= 2 && split <= kSliceWarps;
    int parts = 1;
    if (sliced) {
        while ((1 << p.slice_log2) < split) ++p.slice_log2;
        p.k_per_slice = (int)round_up((p.K + (1 << p.slice_log2) - 1) >> p.slice_log2, kStageK);
    } else {
        const int64_t tiles = (p.N + kWarpRows * kShareWarps - 1) / (kWarpRows * kShareWarps) * ((M + 8 * tiles_m - 1) / (8 * tiles_m));
        parts = (int)std::max<int64_t>(1, std::min<int64_t>({kMaxCluster, 4 * h->sm_count / tiles, p.K / (2 * kStageK)}));
        p.k_per_slice = (int)round_up((p.K + parts - 1) / parts, kStageK);
        parts = (p.K + p.k_per_slice - 1) / p.k_per_slice;
    }
    p.k_per_block = p.k_per_slice << p.slice_log2;
    const cudaError_t e = sliced         ? launch<kSliceWarps, 1>(p, bf16, aligned, parts, st)
                          : tiles_m == 1 ? launch<kShareWarps, 1>(p, bf16, aligned, parts, st)
                          : tiles_m == 2 ? launch<kShareWarps, 2>(p, bf16, aligned, parts, st)
                                         : launch<kShareWarps, 4>(p, bf16, aligned, parts, st);
    if (e != cudaSuccess) return AWE_ERR_CUDA;
    h->launches += 1;
    return AWE_OK;
}
