// A block's scale and values in 8-bit floating point (e4m3).
//
// With amax the largest magnitude among a block's finite values, the scale is
// the least power of two 2^e (e >= -126) with amax <= 448 * 2^e, and 1 for a
// block without one; q = e4m3(x / scale), to nearest, ties to even.  Dividing
// by a power of two is exact, so each value is rounded once, and the result
// depends on no order of evaluation.  The exponent comes from amax's own bits:
// 448 = 1.75 * 2^8, so the mantissa either fits (<= 1.75) or one more is needed.
// A power of two costs no precision: e4m3 keeps 3 mantissa bits wherever in
// its range the block lies, and the block's largest value is in [224, 448].
// e4m3 has no infinity: a non-finite value becomes NaN, so that a corrupted
// activation still reaches the outputs instead of being clipped to 448.
#pragma once

#include "ops_common.cuh"

namespace ct {
namespace ops {
namespace {

// magnitude bits of a finite value, 0 for a non-finite one: ordered like the magnitudes
__device__ __forceinline__ uint32_t mag_bits(float v) {
    const uint32_t b = __float_as_uint(v) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? b : 0u;
}

// (scale, 1 / scale), both exact
__device__ __forceinline__ void block_scale(uint32_t amax, float &scale, float &inv) {
    // exponent field, one more when the mantissa exceeds 1.75, less the 8 of 448's exponent
    const int f = max((int)((amax + 0x1FFFFFu) >> 23) - 8, 1);
    scale = amax == 0u ? 1.f : __uint_as_float((uint32_t)f << 23);
    inv = amax == 0u ? 1.f : __uint_as_float((uint32_t)(254 - f) << 23);
}

// two e4m3 values, `lo` in the low byte; NaN for a non-finite input (x * 0 is
// NaN there and 0 elsewhere; the conversion alone would make 448 of infinity)
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi, float inv) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(fmaf(hi, 0.f, hi * inv)), "f"(fmaf(lo, 0.f, lo * inv)));
    return r;
}

// The largest magnitude of 16 bytes of values, as FP32 bits; where one is not
// finite some value from 0x7F800000 on, or what the finite ones give.
template <typename T> __device__ __forceinline__ uint32_t largest_any(const uint4 &u);
template <> __device__ __forceinline__ uint32_t largest_any<float>(const uint4 &u) {
    return max(max(u.x & 0x7FFFFFFFu, u.y & 0x7FFFFFFFu), max(u.z & 0x7FFFFFFFu, u.w & 0x7FFFFFFFu));
}
template <> __device__ __forceinline__ uint32_t largest_any<__half>(const uint4 &u) {
    // magnitudes as 16-bit integers are ordered like the values
    const uint32_t m = __vmaxu2(__vmaxu2(u.x & 0x7FFF7FFFu, u.y & 0x7FFF7FFFu), __vmaxu2(u.z & 0x7FFF7FFFu, u.w & 0x7FFF7FFFu));
    return __float_as_uint(__half2float(__ushort_as_half((unsigned short)max(m & 0xFFFFu, m >> 16))));
}
template <> __device__ __forceinline__ uint32_t largest_any<__nv_bfloat16>(const uint4 &u) {
    const uint32_t m = __vmaxu2(__vmaxu2(u.x & 0x7FFF7FFFu, u.y & 0x7FFF7FFFu), __vmaxu2(u.z & 0x7FFF7FFFu, u.w & 0x7FFF7FFFu));
    return max(m & 0xFFFFu, m >> 16) << 16;
}

template <typename T, int V> __device__ __forceinline__ uint32_t largest(const uint4 &u) {
    float v[V];
    unpack16<T>(u, v);
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) amax = max(amax, mag_bits(v[i]));
    return amax;
}

// 16 bytes of values as V bytes
template <typename T, int V> __device__ __forceinline__ void convert(const uint4 &u, float inv, uint32_t (&w)[V / 4]) {
    float v[V];
    unpack16<T>(u, v);
#pragma unroll
    for (int i = 0; i < V / 4; ++i)
        w[i] = e4m3x2(v[4 * i], v[4 * i + 1], inv) | (e4m3x2(v[4 * i + 2], v[4 * i + 3], inv) << 16);
}

}  // namespace
}  // namespace ops
}  // namespace ct
