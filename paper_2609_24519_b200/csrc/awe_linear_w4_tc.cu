// Linear layer with 4-bit weights on tcgen05: the weights, unpacked to 16-bit integers, pass through tensor memory.
//
// The formula is that of awe_linear_w4.cu.  Here the matrix instruction's M = 128 rows are rows of the weight and its
// N columns kMt rows of x.  Codes are unpacked in registers and stored to tensor memory, where the instruction
// reads its first operand, so that only x takes shared-memory bandwidth (with both operands there, writing and reading
// them would cost twice what the product does).  Thread = row of the weight on the way in and on the way out: a group's
// sum comes back from tensor memory, is multiplied with the row's scale and added in registers.
//
// Eight warps unpack, eight drain, one thread issues the copies (TMA), one the products; what they wait for is counted in
// stages of 256 k, or in as many groups as half of the accumulator columns hold.  Up to 8 blocks along K form a cluster and
// add their sums through each other's shared memory in a fixed order.
#include <cooperative_groups.h>
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "gemm_common.cuh"
#include "linear_w4.cuh"
#include "ptx_serve.cuh"

namespace awe {
namespace {

using namespace serve;

constexpr int kRowsN = 128;
constexpr int kStageK = 256;
constexpr int kUnpackers = 8, kDrainers = 8;  // warps, in this order, then the copying and the multiplying one
constexpr int kCopier = kUnpackers + kDrainers, kMultiplier = kCopier + 1;
constexpr int kThreads = 32 * (kMultiplier + 1);
constexpr int kTmemCols = 512;
constexpr int kAccCols = 128;           // columns of one of the two sets of accumulators
constexpr int kABuffers = 2;            // stages of unpacked codes in tensor memory
constexpr int kACols = kStageK / 2;     // two values per column
constexpr int kCodesPitch = kStageK / 2 + 16;  // bytes per row where rows are copied piece by piece
constexpr int kMaxCluster = 8;
constexpr int kSlabStages = 4;          // stages whose scales and zero points are copied together
constexpr int kSlabK = kSlabStages * kStageK;

struct TcParams {
    const uint8_t* codes;
    const uint8_t *scale, *zero;
    const void* x;
    void* y;
    int64_t row_bytes, ldx, ldy;
    int M, N, K, group_log2, groups, k_per_block;
    int scale_bf16, y_f32, x_tma;
    int scale_pitch, zero_pitch;  // bytes of a row's scales and zero points of a slab, with room for what an unaligned row spills over
    unsigned int* status;
};

template <int kMt, bool kAligned>
struct Config {
    static constexpr int kStages = kMt == 128 ? 2 : (kMt == 64 ? 3 : 4);
    static constexpr int kXBytes = kMt * kStageK * 2;
    static constexpr int kCodesBytes = kRowsN * (kAligned ? kStageK / 2 : kCodesPitch);
    static constexpr int kStageBytes = kXBytes + kCodesBytes;
    static constexpr int kRingBytes = kStages * kStageBytes;
    static constexpr int kSumBytes = kMt * kRowsN * 4;
    static constexpr int kSlabBytes = kRowsN * (80 + 48);  // for groups of 32
    static constexpr int kBehindBytes = kMt * 16;  // the 33rd piece of a row of x that does not start on 16 bytes
    static constexpr int kSlabAt = kRingBytes > kSumBytes ? kRingBytes : kSumBytes;
    static constexpr int kNeeded = 1024 + kSlabAt + 2 * kSlabBytes + kBehindBytes + 512;
    // A block takes all of tensor memory: a second one on the SM would wait for it while its cluster waits for it.
    static constexpr int kSmemBytes = kNeeded > 120 * 1024 ? kNeeded : 120 * 1024;
    static_assert(kMt <= kAccCols && 2 * kAccCols + kABuffers * kACols <= kTmemCols, "tensor memory");
    static_assert(kStageBytes % 1024 == 0, "swizzled tiles");
    static_assert(kSmemBytes <= 227 * 1024, "shared memory");
};

struct Shared {
    uint64_t full[4], empty[4];             // stage of the ring: copied / read by the workers and the products
    uint64_t x_full[4];                     // x of the stage moved by the draining warps
    uint64_t a_full[kABuffers], a_empty[kABuffers];
    uint64_t acc_full[2], acc_empty[2];
    uint32_t tmem_base;
    volatile uint32_t abort_flag;
};

__device__ __noinline__ bool wait_long(volatile uint32_t* abort_flag, uint32_t bar, uint32_t parity, unsigned int* status, int site) {
    return gemm::bounded_wait_ns(abort_flag, bar, parity, status, site, gemm::kWaitLimitNs);
}
// Position in a ring: slot and the parity of its current round.
template <int kSlots>
struct Turn {
    int slot = 0;
    uint32_t round = 0;
    __device__ __forceinline__ void next() {
        if (++slot == kSlots) slot = 0, round ^= 1;
    }
};

// The eight nibbles of a word as four pairs (0,1), (2,3), ... of 16-bit floats, less the offset.
//   FP16: byte b over 0x64: (1024 + u, 1024 + 16 u') with u = code + 8; times (1, 1/16), less (1032 + z, 72 + z)
//   BF16: nibbles over 0x43: 128 + u, less 136 + z
template <bool kBf16>
__device__ __forceinline__ void unpack_in_order(uint32_t w, uint32_t offset, uint32_t* f) {
    if constexpr (kBf16) {
        const __nv_bfloat162 off = *reinterpret_cast<const __nv_bfloat162*>(&offset);
        const uint32_t w4 = w >> 4;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const uint32_t v = and_xor(__byte_perm(w, w4, 0x4400 + 0x1111 * b), 0x000F000Fu, 0x43084308u);
            const __nv_bfloat162 h = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), off);
            f[b] = *reinterpret_cast<const uint32_t*>(&h);
        }
    } else {
        const __half2 off = *reinterpret_cast<const __half2*>(&offset);
        const uint32_t mul = 0x2C003C00u;  // (1, 1/16)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const uint32_t v = and_xor(__byte_perm(w, 0x64u, 0x4040 + 0x0101 * b), 0xFFF0FF0Fu, 0x00800008u);
            const __half2 h = __hfma2(*reinterpret_cast<const __half2*>(&v), *reinterpret_cast<const __half2*>(&mul), off);
            f[b] = *reinterpret_cast<const uint32_t*>(&h);
        }
    }
}

template <int kMt, bool kBf16, bool kAligned>
__global__ void __launch_bounds__(kThreads, 1)
linear_w4_tc_kernel(const __grid_constant__ CUtensorMap map_codes, const __grid_constant__ CUtensorMap map_x,
                    const __grid_constant__ TcParams p) {
    namespace cg = cooperative_groups;
    using C = Config<kMt, kAligned>;
    constexpr int kStages = C::kStages, kCols = kMt / 2;  // columns a worker drains
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = ptx::smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base - raw);
    Shared* sh = reinterpret_cast<Shared*>(smem + C::kSlabAt + 2 * C::kSlabBytes + C::kBehindBytes);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int n0 = blockIdx.x * kRowsN, m0 = blockIdx.z * kMt, k0 = blockIdx.y * p.k_per_block;
    const int k1 = min(p.K, k0 + p.k_per_block), n_stages = k1 > k0 ? (k1 - k0 + kStageK - 1) / kStageK : 0;
    const int per_stage = p.group_log2 >= 8 ? 1 : kStageK >> p.group_log2;  // groups of a stage, or part of one
    const int per_set = min(per_stage, kAccCols / kMt), sets = per_stage / per_set;

    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            ptx::mbar_init(ptx::smem_u32(&sh->full[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&sh->empty[s]), kUnpackers + 1);
            ptx::mbar_init(ptx::smem_u32(&sh->x_full[s]), kDrainers);
        }
        for (int s = 0; s < kABuffers; ++s) {
            ptx::mbar_init(ptx::smem_u32(&sh->a_full[s]), kUnpackers);
            ptx::mbar_init(ptx::smem_u32(&sh->a_empty[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(ptx::smem_u32(&sh->acc_full[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&sh->acc_empty[s]), kDrainers);
        }
        sh->abort_flag = 0;
        ptx::fence_mbar_init();
        if (kAligned) ptx::prefetch_tensormap(&map_codes);
        if (p.x_tma) ptx::prefetch_tensormap(&map_x);
    }
    if (warp == kMultiplier) {
        ptx::tmem_alloc(ptx::smem_u32(&sh->tmem_base), kTmemCols);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = sh->tmem_base, tmem_a = tmem + 2 * kAccCols;
    auto wait = [&](uint64_t& bar, uint32_t parity, int site) {
        const uint32_t at = ptx::smem_u32(&bar);
        return ptx::mbar_try_wait(at, parity) || wait_long(&sh->abort_flag, at, parity, p.status, site);
    };
    auto x_of = [&](int slot) { return base + slot * C::kStageBytes; };
    auto codes_of = [&](int slot) { return x_of(slot) + C::kXBytes; };
    auto slab_of = [&](int j) { return base + C::kSlabAt + (j & 1) * C::kSlabBytes; };  // scales, then zero points

    cg::cluster_group cluster = cg::this_cluster();
    const int parts = (int)cluster.num_blocks(), rows_m = min(kMt, p.M - m0);
    float* sums = reinterpret_cast<float*>(smem);  // in the ring's place, once the last products are complete
    auto store = [&](int m, int n, float v) {
        const int64_t at = (int64_t)(m0 + m) * p.ldy + n0 + n;
        if (p.y_f32) reinterpret_cast<float*>(p.y)[at] = v;
        else reinterpret_cast<typename Half<kBf16>::type*>(p.y)[at] = Half<kBf16>::from_float(v);
    };

    if (warp == kCopier) {  // ---- copies
        if (lane == 0 && (kAligned || p.x_tma)) {
            const uint32_t bytes = (kAligned ? C::kCodesBytes : 0) + (p.x_tma ? C::kXBytes : 0);
            Turn<kStages> at;
            int i = 0;
            for (; i < n_stages; ++i, at.next()) {
                if (!wait(sh->empty[at.slot], at.round ^ 1, 20)) break;
                const uint32_t bar = ptx::smem_u32(&sh->full[at.slot]);
                ptx::mbar_arrive_expect_tx(bar, bytes);
                const int k = k0 + i * kStageK;
                if (kAligned) ptx::tma_load_2d(codes_of(at.slot), &map_codes, bar, k / 2, n0);
                if (p.x_tma)
                    for (int c = 0; c < 4; ++c) ptx::tma_load_2d(x_of(at.slot) + c * kMt * 128, &map_x, bar, k + 64 * c, m0);
            }
            if (i < n_stages)  // given up: no copy may land after the block has left
                for (int j = max(0, i - kStages); j < i; ++j)
                    for (int tries = 0; tries < (1 << 20) && !ptx::mbar_try_wait(ptx::smem_u32(&sh->full[j % kStages]), (j / kStages) & 1); ++tries) {
                    }
        }
    } else if (warp == kMultiplier) {  // ---- products
        if (lane == 0) {
            constexpr uint32_t kIdesc = (1u << 4) | ((kBf16 ? 1u : 0u) << 7) | ((kBf16 ? 1u : 0u) << 10) | ((uint32_t)(kMt >> 3) << 17) | (8u << 24);
            Turn<kStages> at;
            Turn<kABuffers> a;
            Turn<2> acc;
            bool ok = true;
            // The products of a stage whose groups are kSteps of the instruction's 16 k, all of it unrolled: a loop that
            // computes descriptors and flags takes longer per product than the product.
            auto issue = [&](auto steps_c) {
                constexpr int kSteps = decltype(steps_c)::value, kGroups = kStageK / 16 / kSteps;
                constexpr int kSet = kGroups < kAccCols / kMt ? kGroups : kAccCols / kMt;
                const uint64_t desc = ptx::smem_desc_k_sw128(x_of(at.slot));
                const uint32_t from = tmem_a + a.slot * kACols;
#pragma unroll
                for (int set = 0; set < kGroups / kSet; ++set, acc.next()) {
                    if (!(ok = ok && wait(sh->acc_empty[acc.slot], acc.round ^ 1, 23))) return;
                    ptx::tc_fence_after();
                    const uint32_t to = tmem + acc.slot * kAccCols;
#pragma unroll
                    for (int e = 0; e < kSet * kSteps; ++e) {
                        const int c = set * kSet * kSteps + e;
                        ptx::mma_f16_ta(to + e / kSteps * kMt, from + c * 8, desc + ((c >> 2) * kMt * 128 + (c & 3) * 32) / 16, kIdesc, e % kSteps != 0);
                    }
                    ptx::mma_commit(ptx::smem_u32(&sh->acc_full[acc.slot]));
                }
            };
            for (int i = 0; i < n_stages && ok; ++i, at.next(), a.next()) {
                if (kAligned || p.x_tma) ok = wait(sh->full[at.slot], at.round, 21);
                if (!p.x_tma) ok = ok && wait(sh->x_full[at.slot], at.round, 28);
                ok = ok && wait(sh->a_full[a.slot], a.round, 22);
                if (!ok) break;
                ptx::tc_fence_after();
                if (per_stage == 1) issue(std::integral_constant<int, 16>());
                else if (per_stage == 2) issue(std::integral_constant<int, 8>());
                else if (per_stage == 4) issue(std::integral_constant<int, 4>());
                else issue(std::integral_constant<int, 2>());
                ptx::mma_commit(ptx::smem_u32(&sh->empty[at.slot]));
                ptx::mma_commit(ptx::smem_u32(&sh->a_empty[a.slot]));
            }
        }
    } else if (warp < kUnpackers) {  // ---- unpack: row 32 q + lane of the weight, half of a stage's k
        const int q = warp & 3, half = warp >> 2, row = 32 * q + lane, n = min(n0 + row, p.N - 1);
        const uint32_t lanes = (uint32_t)(32 * q) << 16;
        const int64_t row_groups = (int64_t)n * p.groups;
        const int shift = kAligned ? 0 : (int)((uintptr_t)(p.codes + (int64_t)n * p.row_bytes + (k0 >> 1)) & 15);
        auto copy_codes = [&](int i) {  // 9 pieces per row, 16 threads at a row
            if (i < n_stages && (tid & 15) < 9) {
                const int k = k0 + i * kStageK, bytes = (min(k1 - k, kStageK) + 1) >> 1;
                const uint32_t to = codes_of(i % kStages);
#pragma unroll 2
                for (int r = tid >> 4; r < kRowsN; r += 2 * kUnpackers)
                    copy_piece(to + r * kCodesPitch, p.codes + (int64_t)min(n0 + r, p.N - 1) * p.row_bytes + (k >> 1), bytes, tid & 15, p.codes);
            }
            cp_async_commit();
        };
        auto copy_zeros = [&](int j) {  // of slab j, two threads per row
            const int k = k0 + j * kSlabK, r = tid >> 1;
            if (k >= k1) return;
            const int first = k >> p.group_log2, n_groups = ((min(k1, k + kSlabK) - 1) >> p.group_log2) + 1 - first;
            for (int c = tid & 1; 16 * c < p.zero_pitch; c += 2)
                copy_piece(slab_of(j) + kRowsN * p.scale_pitch + r * p.zero_pitch, p.zero + (int64_t)min(n0 + r, p.N - 1) * p.groups + first, n_groups, c, p.zero);
        };
        uint32_t zero_row = 0;  // where this row's zero point of group 0 of the matrix would stand
        Turn<kStages> at;
        Turn<kABuffers> a;
        bool ok = true;
        copy_zeros(0);
        if (kAligned) cp_async_commit();
        else
            for (int i = 0; i < kStages - 1; ++i) copy_codes(i);
        for (int i = 0; i < n_stages; ++i, at.next(), a.next()) {
            const bool slab_begins = i % kSlabStages == 0 && p.zero;
            if (!kAligned || slab_begins) {
                // the slab's copies are as old as the slab before, or came with the first stage's
                cp_async_wait<kAligned ? 0 : kStages - 2>();
                asm volatile("bar.sync 1, %0;" ::"n"(32 * kUnpackers) : "memory");
                if (slab_begins) {
                    const int j = i / kSlabStages, first = (k0 + j * kSlabK) >> p.group_log2;
                    zero_row = slab_of(j) + kRowsN * p.scale_pitch + row * p.zero_pitch + ((uint32_t)(uintptr_t)(p.zero + row_groups + first) & 15) - first;
                    copy_zeros(j + 1);
                    if (kAligned) cp_async_commit();
                }
                if (!kAligned) copy_codes(i + kStages - 1);
            }
            if (!ok) continue;  // the others may be waiting at the barrier above
            uint32_t w[16];
            if constexpr (kAligned) {
                ok = __all_sync(~0u, wait(sh->full[at.slot], at.round, 26));
                if (!ok) continue;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint4 v = lds128(codes_of(at.slot) + row * 128 + (((4 * half + j) ^ (row & 7)) << 4));
                    w[4 * j] = v.x, w[4 * j + 1] = v.y, w[4 * j + 2] = v.z, w[4 * j + 3] = v.w;
                }
            } else {
                // 64 bytes from byte `shift` on, out of five pieces
                uint32_t v[20];
#pragma unroll
                for (int j = 0; j < 5; ++j) {
                    const uint4 u = lds128(codes_of(at.slot) + row * kCodesPitch + 64 * half + 16 * j);
                    v[4 * j] = u.x, v[4 * j + 1] = u.y, v[4 * j + 2] = u.z, v[4 * j + 3] = u.w;
                }
                if (shift & 8)
#pragma unroll
                    for (int j = 0; j < 18; ++j) v[j] = v[j + 2];
                if (shift & 4)
#pragma unroll
                    for (int j = 0; j < 17; ++j) v[j] = v[j + 1];
#pragma unroll
                for (int j = 0; j < 16; ++j) w[j] = __funnelshift_r(v[j], v[j + 1], 8 * (shift & 3));
            }
            const int k = k0 + i * kStageK + 128 * half;
            uint32_t u[4] = {0, 0, 0, 0};  // zero point + 8 of each 32 k
            if (p.zero) {
#pragma unroll
                for (int j = 0; j < 4; ++j) asm volatile("ld.shared.u8 %0, [%1];" : "=r"(u[j]) : "r"(zero_row + ((k + 32 * j) >> p.group_log2)));
            }
            ok = __all_sync(~0u, wait(sh->a_empty[a.slot], a.round ^ 1, 27));
            if (!ok) continue;
            ptx::tc_fence_after();
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                uint32_t f[32];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t z = (u[2 * part + j] & 15) ^ 8, off = kBf16 ? 0x43004300u + z * 0x10001u : 0xD400E400u + z * 0x100001u;
#pragma unroll
                    for (int c = 0; c < 4; ++c) unpack_in_order<kBf16>(w[8 * part + 4 * j + c], off, f + 16 * j + 4 * c);
                }
                ptx::tmem_st_32x32(tmem_a + lanes + a.slot * kACols + 64 * half + 32 * part, f);
            }
            ptx::tmem_wait_st();
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                ptx::mbar_arrive(ptx::smem_u32(&sh->a_full[a.slot]));
                ptx::mbar_arrive(ptx::smem_u32(&sh->empty[at.slot]));
            }
        }
        cp_async_wait<0>();
    } else {  // ---- drain: row 32 q + lane of the weight, half of the columns
        const int q = warp & 3, half = (warp - kUnpackers) >> 2, row = 32 * q + lane, thread = tid - 32 * kUnpackers;
        const uint32_t lanes = (uint32_t)(32 * q) << 16;
        const int64_t row_groups = (int64_t)min(n0 + row, p.N - 1) * p.groups;
        auto copy_scales = [&](int j) {  // of slab j, two threads per row
            const int k = k0 + j * kSlabK, r = thread >> 1;
            if (k >= k1) return;
            const int first = k >> p.group_log2, n_groups = ((min(k1, k + kSlabK) - 1) >> p.group_log2) + 1 - first;
            for (int c = thread & 1; 16 * c < p.scale_pitch; c += 2)
                copy_piece(slab_of(j) + r * p.scale_pitch, p.scale + 2 * ((int64_t)min(n0 + r, p.N - 1) * p.groups + first), 2 * n_groups, c, p.scale);
        };
        float total[kCols];
#pragma unroll
        for (int c = 0; c < kCols; ++c) total[c] = 0.0f;
        uint32_t scale_row[2] = {0, 0};  // where this row's scale of group 0 of the matrix would stand, by the slab's parity
        Turn<2> acc;
        bool ok = true;
        // x where TMA cannot read it: a warp copies the 16-byte pieces that 256 k of a row touch to the places of the
        // row's own pieces, and shifts them there once they have come.
        const uint32_t behind = base + C::kSlabAt + 2 * C::kSlabBytes;
        const int first_m = warp - kUnpackers;  // this warp's rows: first_m, first_m + 8, ...
        const int64_t row_step = 2 * kDrainers * p.ldx;
        const uint8_t *x0 = reinterpret_cast<const uint8_t*>(p.x), *x1 = x0 + 2 * ((int64_t)(p.M - 1) * p.ldx + p.K);
        const uint8_t* x_row = x0 + 2 * ((int64_t)(m0 + first_m) * p.ldx + k0);
        const uint32_t x_place = (lane >> 3) * kMt * 128 + first_m * 128 + (((lane & 7) ^ (first_m & 7)) << 4);  // in a slot
        const uint32_t x_next = lane == 31 ? 0 : ((lane + 1) >> 3) * kMt * 128 + first_m * 128 + ((((lane + 1) & 7) ^ (first_m & 7)) << 4);
        auto copy_x = [&](int i) {  // the products of the stage that had this slot have been drained
            if (i < n_stages) {
                const uint8_t* at = x_row + 2 * i * kStageK;
                uint32_t to = x_of(i % kStages) + x_place, to_behind = behind + 16 * first_m;
                // nothing in front of x or behind it is read
                const bool inside = x_row + 2 * i * kStageK - 16 >= x0 && x0 + 2 * ((int64_t)(m0 + rows_m - 1) * p.ldx + k0 + (i + 1) * kStageK) + 32 <= x1;
#pragma unroll 4
                for (int m = first_m; m < rows_m; m += kDrainers, at += row_step, to += 128 * kDrainers, to_behind += 16 * kDrainers) {
                    const uint8_t *row0 = reinterpret_cast<const uint8_t*>((uintptr_t)at & ~(uintptr_t)15), *from = row0 + 16 * lane;
                    if (inside) {
                        cp_async16(to, from, 16);
                        if (lane == 31) cp_async16(to_behind, from + 16, 16);
                    } else {
                        const int64_t left = x1 - from;
                        if (from >= x0) cp_async16(to, left > 0 ? from : row0, (uint32_t)min((int64_t)16, max((int64_t)0, left)));
                        else copy_first_piece(to, from, (int)(x0 - from), (int)min((int64_t)16, left));
                        if (lane == 31) cp_async16(to_behind, left > 16 ? from + 16 : row0, (uint32_t)min((int64_t)16, max((int64_t)0, left - 16)));
                    }
                }
            }
            cp_async_commit();
        };
        auto shift_x = [&](int i) {
            const int n_k = k1 - k0 - i * kStageK;
            const uint32_t slot = x_of(i % kStages);
            constexpr int kBatch = 4;  // rows whose latencies overlap
            uint32_t at = (uint32_t)(uintptr_t)x_row + 2 * i * kStageK;  // only its low bits count
#pragma unroll 1
            for (int r0 = 0; r0 < kMt / kDrainers; r0 += kBatch) {
                uint4 v[kBatch], u[kBatch];
#pragma unroll
                for (int r = 0; r < kBatch; ++r) {
                    const uint32_t off = (r0 + r) * kDrainers * 128;
                    v[r] = lds128(slot + x_place + off);
                    u[r] = lds128(lane == 31 ? behind + 16 * (first_m + (r0 + r) * kDrainers) : slot + x_next + off);
                }
                __syncwarp();
#pragma unroll
                for (int r = 0; r < kBatch; ++r, at += (uint32_t)row_step) {
                    const bool live = first_m + (r0 + r) * kDrainers < rows_m;
                    uint32_t w[8] = {v[r].x, v[r].y, v[r].z, v[r].w, u[r].x, u[r].y, u[r].z, u[r].w};
                    if (at & 8) {
#pragma unroll
                        for (int j = 0; j < 6; ++j) w[j] = w[j + 2];
                    }
                    if (at & 4) {
#pragma unroll
                        for (int j = 0; j < 5; ++j) w[j] = w[j + 1];
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = live ? __funnelshift_r(w[j], w[j + 1], 8 * (at & 2)) : 0u;
                    if (n_k < kStageK) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int left = n_k - 8 * lane - 2 * j;
                            w[j] = left >= 2 ? w[j] : (left == 1 ? w[j] & 0xFFFFu : 0u);
                        }
                    }
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(slot + x_place + (r0 + r) * kDrainers * 128), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3])
                                 : "memory");
                }
            }
            ptx::fence_proxy_async();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh->x_full[i % kStages]));
        };
        auto drain = [&](int i) {  // the groups of stage i
            uint32_t scale_at = (i / kSlabStages & 1 ? scale_row[1] : scale_row[0]) + 2 * ((k0 + i * kStageK) >> p.group_log2);
            for (int set = 0; set < sets; ++set, acc.next()) {
                ok = __all_sync(~0u, ok && wait(sh->acc_full[acc.slot], acc.round, 24));
                if (!ok) break;
                ptx::tc_fence_after();
                uint32_t from = tmem + lanes + acc.slot * kAccCols + half * kCols;
#pragma unroll 2
                for (int j = 0; j < per_set; ++j, scale_at += 2, from += kMt) {
                    constexpr int kBlock = kCols == 32 || kCols == 16 ? 16 : 8;
                    uint32_t rs;
                    asm volatile("ld.shared.u16 %0, [%1];" : "=r"(rs) : "r"(scale_at));
                    const float s = p.scale_bf16 ? __uint_as_float(rs << 16) : __half2float(__ushort_as_half((unsigned short)rs));
                    uint32_t v[2][kBlock];
                    auto load = [&](int c) {
                        if constexpr (kBlock == 8) ptx::tmem_ld_32x8(from + c, v[(c / kBlock) & 1]);
                        else ptx::tmem_ld_32x16(from + c, v[(c / kBlock) & 1]);
                    };
                    load(0);
#pragma unroll
                    for (int c = 0; c < kCols; c += kBlock) {
                        ptx::tmem_wait_ld();
                        if (c + kBlock < kCols) load(c + kBlock);
#pragma unroll
                        for (int e = 0; e < kBlock; ++e) total[c + e] = fmaf(__uint_as_float(v[(c / kBlock) & 1][e]), s, total[c + e]);
                    }
                }
                gemm::release(ptx::smem_u32(&sh->acc_empty[acc.slot]), lane, false);
            }
        };
        copy_scales(0);
        cp_async_commit();
        if (!p.x_tma) copy_x(0);
        for (int i = 0; i < n_stages; ++i) {
            if (!p.x_tma || i % kSlabStages == 0) cp_async_wait<0>();
            if (!p.x_tma) {
                __syncwarp();
                shift_x(i);
            }
            if (i > 0) drain(i - 1);
            if (!p.x_tma) copy_x(i + 1);
            if (i % kSlabStages == 0) {
                const int j = i / kSlabStages, first = (k0 + j * kSlabK) >> p.group_log2;
                asm volatile("bar.sync 2, %0;" ::"n"(32 * kDrainers) : "memory");  // slab j has come, slab j - 1 is done with
                scale_row[j & 1] = slab_of(j) + row * p.scale_pitch + ((uint32_t)(uintptr_t)(p.scale + 2 * (row_groups + first)) & 15) - 2 * first;
                copy_scales(j + 1);
                cp_async_commit();
            }
        }
        if (n_stages) drain(n_stages - 1);
        cp_async_wait<0>();
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
            const int m = half * kCols + c;
            if (m >= rows_m) continue;
            if (parts > 1) sums[m * kRowsN + row] = total[c];
            else if (n0 + row < p.N) store(m, row, total[c]);
        }
    }

    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    if (warp == kMultiplier) ptx::tmem_dealloc(tmem, kTmemCols);
    if (parts == 1) return;
    // ---- the sums of the cluster's blocks, in a fixed order
    const int rank = (int)cluster.block_rank();
    cluster.sync();
    const float4* from[kMaxCluster];
#pragma unroll
    for (int r = 0; r < kMaxCluster; ++r) from[r] = reinterpret_cast<const float4*>(r < parts ? cluster.map_shared_rank(sums, r) : sums);
    const int quads = rows_m * (kRowsN / 4);  // four neighbouring rows of the weight at a time
    const bool vec = !p.y_f32 && ((uintptr_t)p.y & 7) == 0 && (p.ldy & 3) == 0 && n0 + kRowsN <= p.N;
    for (int j = rank * kThreads + tid; j < quads; j += parts * kThreads) {
        float4 part[kMaxCluster];
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r)
            if (r < parts) part[r] = from[r][j];
        float4 v = part[0];
#pragma unroll
        for (int r = 1; r < kMaxCluster; ++r)
            if (r < parts) v.x += part[r].x, v.y += part[r].y, v.z += part[r].z, v.w += part[r].w;
        const int m = j / (kRowsN / 4), n = j % (kRowsN / 4) * 4;
        if (vec) {
            *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(p.y) + (int64_t)(m0 + m) * p.ldy + n0 + n) =
                make_uint2(Half<kBf16>::pack(v.x, v.y), Half<kBf16>::pack(v.z, v.w));
        } else {
            const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (n0 + n + c < p.N) store(m, n + c, e[c]);
        }
    }
    cluster.sync();  // no block leaves while its sums are read
}

awe_status_t make_map_2d(awe_ctx* h, const void* at, bool bytes, int64_t inner, int64_t rows, int64_t pitch, int box_inner, int box_rows,
                         CUtensorMapSwizzle swizzle, CUtensorMap* out) {
    if (!h->encode_tiled) return AWE_ERR_CUDA;
    cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)pitch};
    cuuint32_t box[2] = {(cuuint32_t)box_inner, (cuuint32_t)box_rows}, ones[2] = {1, 1};
    const CUresult r = ((gemm::EncodeTiledFn)h->encode_tiled)(
        out, bytes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void*>(at), dims, strides, box, ones,
        CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? AWE_OK : AWE_ERR_CUDA;
}

template <int kMt, bool kBf16, bool kAligned>
awe_status_t launch(awe_ctx* h, const CUtensorMap& mc, const CUtensorMap& mx, TcParams p, cudaStream_t st) {
    using C = Config<kMt, kAligned>;
    static std::atomic<uint64_t> done{0};
    if (allow_smem(linear_w4_tc_kernel<kMt, kBf16, kAligned>, C::kSmemBytes, h->device, done) != cudaSuccess) return AWE_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = C::kSmemBytes;
    cfg.stream = st;
    cudaLaunchAttribute attr = {};
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    // Parts of K: as many as leave every tile's cluster resident at once, with two stages per block at least.  Fewer clusters of 8
    // fit than the SMs have room for (128 blocks in 16 clusters of 8 take 20 us where 16 of 4 take 12), so the runtime is
    // asked, once per size.
    const dim3 tiles((p.N + kRowsN - 1) / kRowsN, 1, (p.M + kMt - 1) / kMt);
    static std::atomic<int> fit[64][kMaxCluster + 1];  // by device: clusters of each size that are resident at once, plus 1
    int parts = std::max(1, std::min(kMaxCluster, p.K / (2 * kStageK)));
    for (; parts > 1; --parts) {
        if ((int64_t)tiles.x * tiles.z * parts > h->sm_count) continue;
        int n = fit[h->device & 63][parts].load(std::memory_order_relaxed) - 1;
        if (n < 0) {
            attr = cluster_attribute(parts);
            cfg.gridDim = dim3(1, parts, 1);
            if (cudaOccupancyMaxActiveClusters(&n, linear_w4_tc_kernel<kMt, kBf16, kAligned>, &cfg) != cudaSuccess) return AWE_ERR_CUDA;
            fit[h->device & 63][parts].store(n + 1, std::memory_order_relaxed);
        }
        if ((int64_t)tiles.x * tiles.z <= n) break;
    }
    p.k_per_block = (int)round_up((p.K + parts - 1) / parts, kStageK);
    parts = (p.K + p.k_per_block - 1) / p.k_per_block;
    attr = cluster_attribute(parts);
    cfg.gridDim = dim3(tiles.x, parts, tiles.z);
    if (cudaLaunchKernelEx(&cfg, linear_w4_tc_kernel<kMt, kBf16, kAligned>, mc, mx, p) != cudaSuccess) return AWE_ERR_CUDA;
    h->launches += 1;
    return AWE_OK;
}
template <int kMt>
awe_status_t launch(awe_ctx* h, const CUtensorMap& mc, const CUtensorMap& mx, const TcParams& p, bool bf16, bool aligned, cudaStream_t st) {
    if (bf16) return aligned ? launch<kMt, true, true>(h, mc, mx, p, st) : launch<kMt, true, false>(h, mc, mx, p, st);
    return aligned ? launch<kMt, false, true>(h, mc, mx, p, st) : launch<kMt, false, false>(h, mc, mx, p, st);
}

}  // namespace

awe_status_t linear_w4_tc(awe_ctx* h, const awe_w4_matrix& W, const void* x, bool bf16, int64_t M, int64_t ldx, void* y, bool y_f32,
                          int64_t ldy, cudaStream_t st) {
    TcParams p = {};
    p.codes = (const uint8_t*)W.codes_dev, p.scale = (const uint8_t*)W.scale_dev, p.zero = (const uint8_t*)W.zero_dev, p.x = x, p.y = y;
    p.row_bytes = W.ld / 2, p.ldx = ldx, p.ldy = ldy;
    p.M = (int)M, p.N = (int)W.N, p.K = (int)W.K;
    while ((int64_t)1 << p.group_log2 < W.group && p.group_log2 < 31) ++p.group_log2;
    p.groups = (int)((W.K + W.group - 1) / W.group);
    p.scale_bf16 = W.scale_type == AWE_BF16, p.y_f32 = y_f32;
    p.x_tma = (uintptr_t)x % 16 == 0 && ldx % 8 == 0;
    const int slab_groups = std::max(1, kSlabK >> p.group_log2);
    p.scale_pitch = (int)round_up(2 * slab_groups, 16) + 16;
    p.zero_pitch = p.zero ? (int)round_up(slab_groups, 16) + 16 : 0;
    p.status = h->status_dev;
    const bool aligned = (uintptr_t)W.codes_dev % 16 == 0 && W.ld % 32 == 0;
    // Above 64 rows the taller tile unpacks a weight once for 128 rows, and pays once its tiles are many: 8,192 x 8,192 for 128
    // rows 41 us against 47 with 64, but 2,048 x 4,096 28 against 13.
    int mt = M <= 32 ? 32 : 64;
    if (M > 64 && (W.N + kRowsN - 1) / kRowsN * ((M + 127) / 128) > 32) mt = 128;
    CUtensorMap mc = {}, mx = {};
    awe_status_t s;
    if (aligned && (s = make_map_2d(h, W.codes_dev, true, (W.K + 1) / 2, W.N, W.ld / 2, kStageK / 2, kRowsN, CU_TENSOR_MAP_SWIZZLE_128B, &mc)) != AWE_OK)
        return s;
    if (p.x_tma && (s = make_map_2d(h, x, false, W.K, M, 2 * ldx, 64, mt, CU_TENSOR_MAP_SWIZZLE_128B, &mx)) != AWE_OK)
        return s;
    switch (mt) {
        case 32: return launch<32>(h, mc, mx, p, bf16, aligned, st);
        case 64: return launch<64>(h, mc, mx, p, bf16, aligned, st);
        default: return launch<128>(h, mc, mx, p, bf16, aligned, st);
    }
}

}  // namespace awe
