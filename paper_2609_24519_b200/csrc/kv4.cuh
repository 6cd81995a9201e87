// The paged 4-bit cache's format, shared by the kernels that write and read it.
//
// Parameter word of a token and head: FP16 of 16 * scale, its lowest four bits replaced by the zero point.  A scale has 7
// significant bits and a code less its zero point is at most 15, so scale * (code - zero) has 11: FP16 holds it.  The smallest scale is
// 2^-18 (its 7th bit is FP16's smallest subnormal), the largest 4,064 (the largest 7-bit FP16 over 16; 15 times it is below 65,504).
#pragma once
#include "awe_internal.h"
#include "serve_common.cuh"

namespace awe {

constexpr float kKv4LeastScale = 3.814697265625e-6f, kKv4MostScale = 4064.0f;
constexpr float kKv4MostValue = 30480.0f;  // 7.5 times the largest scale: a range inside these ends has a scale that is not above it

// Scale of a parameter word.  Any word gives a finite positive one: a NaN pattern the smallest.
__device__ __forceinline__ float kv4_scale(uint32_t word) {
    const float s = __half2float(__ushort_as_half((unsigned short)(word & 0xFFF0u))) * 0.0625f;
    return fminf(fmaxf(s, kKv4LeastScale), kKv4MostScale);
}
// The nibble of a value 0, which is its zero point with the sign bit flipped: nibble ^ 8 of a code less this is code - zero.
__device__ __forceinline__ uint32_t kv4_zero8(uint32_t word) { return (word & 15u) ^ 8u; }

__device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t fma2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t mul2(uint32_t a, __half2 b) {
    const __half2 d = __hmul2(*reinterpret_cast<const __half2*>(&a), b);
    return *reinterpret_cast<const uint32_t*>(&d);
}
// Codes become FP16 by inserting their nibbles, u = nibble ^ 8, into the mantissa of 1024: 1024 + u for those in bits 0 .. 3 of a half
// word, 1024 + 16 u for those in bits 4 .. 7, a sixteenth of which is 64 + u.  What they lose to become code - zero: 1024 + zero8, 64 + zero8.
// All of it is exact.
struct Kv4Zeros {
    uint32_t low, high;
    __device__ __forceinline__ Kv4Zeros(uint32_t words) {  // the parameter words of the two halves
        const uint32_t z = (words & 0x000F000Fu) ^ 0x00080008u;
        low = z | 0x64006400u, high = (z << 4) | 0xD400D400u;
    }
};
__device__ __forceinline__ uint32_t kv4_low_codes(uint32_t w, const Kv4Zeros& z) { return sub2(serve::and_xor(w, 0x000F000Fu, 0x64086408u), z.low); }
__device__ __forceinline__ uint32_t kv4_high_codes(uint32_t w, const Kv4Zeros& z) {
    return fma2(serve::and_xor(w, 0x00F000F0u, 0x64806480u), 0x2C002C00u, z.high);
}

inline awe_status_t check_kv4_cache(const awe_kv4_cache* c) {
    if (!c || !c->k_dev || !c->v_dev || !c->k_param_dev || !c->v_param_dev || c->n_pages <= 0 || c->n_heads <= 0)
        return AWE_ERR_INVALID_ARG;
    if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1))) return AWE_ERR_UNSUPPORTED;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return AWE_ERR_UNSUPPORTED;
    if (c->n_pages > INT32_MAX || c->n_heads > 65535) return AWE_ERR_UNSUPPORTED;
    if ((uintptr_t)c->k_dev % 16 || (uintptr_t)c->v_dev % 16 || (uintptr_t)c->k_param_dev % 16 || (uintptr_t)c->v_param_dev % 16)
        return AWE_ERR_ALIGNMENT;
    return AWE_OK;
}

}  // namespace awe
