// What the two attention kernels share: one for few query rows (awe_kv_attention.cu), one on tcgen05 for many
// (awe_kv_attention_tc.cu).
#pragma once
#include "awe_internal.h"
#include "serve_common.cuh"

namespace awe {

struct AttnParams {
    const int8_t *k, *v;
    const float *k_scale, *v_scale;      // 8 bits: of pages and heads
    const uint16_t *k_param, *v_param;  // 4 bits: of tokens and heads
    const void* q;
    void* out;
    float* lse;
    const int32_t *q_start, *ctx_len, *table;
    int64_t* unit_steps;  // B + 1: exclusive sum over the requests of units x steps
    float* part_vec;      // [2 * blocks][8 * kNT rows][head_dim]
    float4* part_stat;    // [2 * blocks][8 * kNT rows]: reference (base-2 logarithm), sum of the rounded exponentials, sum
    int64_t ldq, ldo, ld_table, T;
    float scale_log2;     // scale / ln 2
    int B, heads, group, page_log2, n_pages, max_pages, causal, blocks;
    int64_t window;
    int whole;            // a block per unit, which nothing cuts
};

// The steps are dealt out to the blocks in order, as evenly as whole numbers go: the first `extra` blocks take one more.
struct Deal {
    int64_t each;
    int extra, blocks;
    __device__ __forceinline__ Deal(int64_t total, int most_blocks) {
        blocks = (int)min((int64_t)most_blocks, max(total, (int64_t)1));
        each = total / blocks;
        extra = (int)(total - each * blocks);
    }
    __device__ __forceinline__ int64_t begin(int i) const { return each * i + min(i, extra); }
    __device__ __forceinline__ int block_of(int64_t step) const {
        const int64_t cut = (each + 1) * extra;
        return step < cut ? (int)(step / (each + 1)) : extra + (int)((step - cut) / each);
    }
};

// Weights are rounded to FP16 as exp2(s - m).  The reference m is put kBelow below the largest s so far and moves only when an s
// passes it by more than kMostAbove, which is rare, so the largest weight lies between 2^10 and 2^15 and FP16 holds all that
// it can beside it: a weight keeps 11 bits down to 2^-24 of the largest, and is off by 2^-35 of that at most below.  (Over the 4-bit cache m
// is a whole number, or moves by whole numbers, so 2^10 is 2^9 there, and 2^-35 is 2^-34.)
constexpr float kBelow = 10.0f, kMostAbove = 15.0f;

// BF16 queries go to FP16 times 2^(15 - e), e the exponent of the row's largest magnitude, whose biased exponent is given: that
// one lands in [2^15, 2^16), and elements down to 2^-32 of it keep all of their 8 bits.  e stays where both powers are normal.
__device__ __forceinline__ int query_exponent(int biased) { return min(max(biased - 127, -111), 127); }
__device__ __forceinline__ float power_of_2(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// Four signed bytes as two pairs of FP16: the byte with its sign bit flipped is u = x + 128, the FP16 pattern
// 0x6400 | u is 1024 + u, and subtracting 1152 is exact.
__device__ __forceinline__ uint32_t bytes_to_half2(uint32_t flipped, uint32_t selector) {
    uint32_t w, h;
    asm("prmt.b32 %0, %1, 0x64646464, %2;" : "=r"(w) : "r"(flipped), "r"(selector));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(h) : "r"(w), "r"(0x64806480u));
    return h;
}
__device__ __forceinline__ uint32_t flip_signs(uint32_t w) { return w ^ 0x80808080u; }  // of four bytes

// Checks the arguments that the two attention entry points share and fills in what they say; `empty`: there is nothing to do.
awe_status_t attention_params(AttnParams& p, bool& empty, const void* q_dev, awe_float_t type, int64_t T, int64_t n_q_heads, int64_t ldq,
                              const int32_t* q_start_dev, const int32_t* ctx_len_dev, int64_t B, const int32_t* block_table_dev,
                              int64_t max_pages, int64_t ld_table, float scale, int causal, int64_t window, void* out_dev, int64_t ldo,
                              float* lse_dev, void* workspace_dev, int64_t n_pages, int64_t n_heads, int64_t page_size, int64_t head_dim);

// Prompts: the tcgen05 kernel, over the cache of 8 bits or of 4; the arguments have been checked, p's pointers into the workspace are not set.
size_t kv_attention_tc_workspace_bytes(awe_ctx* h, int64_t T, int64_t group, int64_t B, int64_t head_dim);
awe_status_t kv_attention_tc(awe_ctx* h, AttnParams p, int64_t head_dim, bool bf16, bool four, void* workspace, cudaStream_t st);

}  // namespace awe
