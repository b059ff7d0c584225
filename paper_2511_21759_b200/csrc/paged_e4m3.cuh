// Codes of 8 bits (e4m3: a sign, four bits of exponent, three behind the first; 0x7f and 0xff are NaN, the largest number is 448) and
// the powers of two that they are scaled by.
#pragma once

#include "paged.cuh"

namespace odb {

namespace {

// 2^e for -126 <= e <= 127
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }
// the exponent of a scale: a power of two from a pool, whatever its memory holds
__device__ __forceinline__ int e4m3_exponent(float scale) {
    return min(max(static_cast<int>(__float_as_uint(scale) >> 23 & 255u) - 127, kPagedLowExp), kPagedHighExp);
}
// the smallest exponent with top <= 448 * 2^e: 448 = 1.75 * 2^8, and a fraction above 1.75 carries into the exponent
__device__ __forceinline__ int e4m3_exponent_for(float top) {
    return min(max(static_cast<int>((__float_as_uint(top) + 0x1fffffu) >> 23) - 127 - 8, kPagedLowExp), kPagedHighExp);
}
// The exponent of the power of two that a row of Q is divided by, from its largest value's bits as bf16: that value is then in 1 .. 2, or, of
// the largest there are, below f16's 2^16, so that the power times a softmax scale stays a number of fp32.  An infinity stays one.
__device__ __forceinline__ int q_exponent(uint32_t top) { return min(max(static_cast<int>(top >> 7) - 127, -126), 112); }
// What a score's product is multiplied by, beyond fp32 its largest number: products that are zero stay zero.
__device__ __forceinline__ float finite_factor(float x) { return fmaxf(fminf(x, 0x1.fffffep127f), -0x1.fffffep127f); }
// two codes, to the nearest even, the first in the low byte; beyond 448 the largest number
__device__ __forceinline__ unsigned short e4m3x2_of(float a, float b) {
    unsigned short r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(r) : "f"(a), "f"(b));
    return r;
}
// the values of two codes, exact, the low byte's in the low half
__device__ __forceinline__ uint32_t f16x2_of(unsigned short codes) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(codes));
    return r;
}
__device__ __forceinline__ uint32_t low_codes(uint32_t w) { return f16x2_of(static_cast<unsigned short>(w)); }
__device__ __forceinline__ uint32_t high_codes(uint32_t w) { return f16x2_of(static_cast<unsigned short>(w >> 16)); }
// some code of the four is NaN: 0x7f + 1 carries into the sign's place
__device__ __forceinline__ bool odd_codes(uint32_t four) { return ((four & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ uint32_t without_nan(uint32_t four) {   // zero in their places
    const uint32_t nan = ((four & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    return four & ~(nan | (nan - (nan >> 7)));
}
__device__ __forceinline__ float2 f32x2_of(unsigned short codes) {
    const uint32_t h = f16x2_of(codes);
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
// four codes times a power of two, rounded again
__device__ __forceinline__ uint32_t e4m3x4_times(uint32_t codes, float by) {
    const float2 a = f32x2_of(static_cast<unsigned short>(codes)), b = f32x2_of(static_cast<unsigned short>(codes >> 16));
    return e4m3x2_of(a.x * by, a.y * by) | static_cast<uint32_t>(e4m3x2_of(b.x * by, b.y * by)) << 16;
}

// a box of rows of the pool
__device__ __forceinline__ void tma_codes(uint32_t dst, const CUtensorMap* tmap, uint64_t* bar, int row) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(tmap)), "r"(smem_u32(bar)), "r"(0), "r"(row)
                 : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
// an arrival once this thread's copies so far have landed; counted among the barrier's.  It says nothing of what the thread has stored itself.
__device__ __forceinline__ void copies_arrive(uint64_t* bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

}  // namespace

}  // namespace odb
