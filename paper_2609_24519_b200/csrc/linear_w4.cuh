// What the two kernels of the 4-bit linear layer share: one on the 16 x 8 x 16 matrix instruction (awe_linear_w4.cu), one
// on tcgen05 with the weights in tensor memory (awe_linear_w4_tc.cu).
#pragma once
#include "awe_internal.h"
#include "serve_common.cuh"

namespace awe {

// The first 16 bytes of an unaligned row whose 16-byte piece begins in front of the array: bytes from `first` on.
static __device__ __noinline__ void copy_first_piece(uint32_t dst, const uint8_t* piece, int first, int bytes) {
    for (int e = 0; e < 16; ++e)
        asm volatile("st.shared.u8 [%0], %1;" ::"r"(dst + e), "r"((uint32_t)(e >= first && e < bytes ? piece[e] : 0)) : "memory");
}
// Piece c of the copy of [src, src + n) to dst + (src mod 16), in pieces of 16 bytes that start on 16-byte boundaries.
// What lies in front of `base` is not ours to read.
__device__ __forceinline__ void copy_piece(uint32_t dst, const uint8_t* src, int n, int c, const uint8_t* base) {
    const int shift = (int)((uintptr_t)src & 15);
    const uint8_t* piece = src - shift + 16 * c;
    const int bytes = min(16, max(0, n + shift - 16 * c));
    if (piece >= base) serve::cp_async16(dst + 16 * c, bytes ? piece : src - shift + 16, bytes);
    else copy_first_piece(dst + 16 * c, piece, (int)(base - piece), bytes);
}
// 8 consecutive 16-bit values of x at any 2-byte alignment.
__device__ __forceinline__ uint4 load_x8(const uint16_t* src, bool vec, int n) {
    uint32_t w[4] = {0, 0, 0, 0};
    if (n >= 8) {
        if (vec) return __ldg(reinterpret_cast<const uint4*>(src));
        if (((uintptr_t)src & 2) == 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = __ldg(reinterpret_cast<const uint32_t*>(src) + e);
        } else {  // the first and the last half word by themselves
            uint32_t v[5];
            v[0] = (uint32_t)__ldg(src) << 16;
#pragma unroll
            for (int e = 0; e < 3; ++e) v[e + 1] = __ldg(reinterpret_cast<const uint32_t*>(src + 1) + e);
            v[4] = __ldg(src + 7);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = __funnelshift_r(v[e], v[e + 1], 16);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) w[e >> 1] |= (uint32_t)src[e] << (16 * (e & 1));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// The product on tcgen05 (M > 16); the arguments have been checked.
awe_status_t linear_w4_tc(awe_ctx* h, const awe_w4_matrix& W, const void* x, bool bf16, int64_t M, int64_t ldx, void* y, bool y_f32,
                          int64_t ldy, cudaStream_t st);

}  // namespace awe
