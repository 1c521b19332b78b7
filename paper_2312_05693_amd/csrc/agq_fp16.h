// fp16 values in float64 arithmetic and back with one rounding, eight at a time, and Eq.2's 8-bit signed grid on them:
// shared by the operators that Section 4.2 keeps in fp16 and by the key/value cache.
#pragma once
#include "agq_device.h"

namespace {

// float64 -> fp16, round to nearest even in ONE step.  The hardware converts
// f64 -> f32 and f32 -> f16; rounding twice to nearest can differ from rounding
// once, so the first step is turned into round-to-odd (truncate, then set the last
// bit when anything was cut off), after which the second rounding is exact: 24
// bits keep two more than the 11 of the target.
__device__ __forceinline__ __half f64_to_f16(double d) {
    float f = (float)d;
    const double back = (double)f;
    if (back != d && fabsf(f) <= 3.0e38f) {   // inexact and not overflowed (NaN compares false)
        uint32_t u = __float_as_uint(f);
        if (fabs(back) > fabs(d)) u -= 1;     // nearest went away from zero: step back to the truncation
        f = __uint_as_float(u | 1u);
    }
    return __float2half_rn(f);
}
__device__ __forceinline__ double h2d(uint16_t h) { return (double)__half2float(__ushort_as_half(h)); }
__device__ __forceinline__ uint16_t d2h(double d) { return __half_as_ushort(f64_to_f16(d)); }

struct Half8 {
    uint16_t v[8];
};
static_assert(sizeof(Half8) == 16, "eight fp16 are one 16-byte access");
__device__ __forceinline__ Half8 load8(const void *p) { return __builtin_bit_cast(Half8, *reinterpret_cast<const uint4 *>(p)); }
__device__ __forceinline__ void store8(void *p, const Half8 &h) { *reinterpret_cast<uint4 *>(p) = __builtin_bit_cast(uint4, h); }

// Eq.2 on one fp16 value, signed 8-bit grid, step 2^e (inv = 2^-e): the product is
// exact in fp32, the rounding is to nearest even.
__device__ __forceinline__ uint32_t quant8_1(uint16_t h, float inv) {
    const float r = rintf(__half2float(__ushort_as_half(h)) * inv);
    return (uint32_t)(int)fminf(fmaxf(r, -128.0f), 127.0f) & 0xFFu;
}
__device__ __forceinline__ uint2 quant8_8(const Half8 &h, float inv) {
    uint2 o;
    o.x = quant8_1(h.v[0], inv) | (quant8_1(h.v[1], inv) << 8) | (quant8_1(h.v[2], inv) << 16) | (quant8_1(h.v[3], inv) << 24);
    o.y = quant8_1(h.v[4], inv) | (quant8_1(h.v[5], inv) << 8) | (quant8_1(h.v[6], inv) << 16) | (quant8_1(h.v[7], inv) << 24);
    return o;
}

}  // namespace
