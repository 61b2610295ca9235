// Device helpers of rows in 8 bits: e4m3 codes with a power of two per block of rows and head.
//
// A scale is the byte b of 2^(b - 127).  It is the smallest with |x| <= 448 * 2^(b - 127) for every finite x of its block, so that
// no code saturates, and a scale that grows moves a code's exponent only: requantising is exact but for codes that fall below the
// smallest normal number.  An infinity has no code: it becomes NaN like NaN itself, and neither has a part in the scale.
#pragma once
#include "gs_train.cuh"

namespace gs {

// Magnitude of x as an integer that orders like it; 0 for what is not finite.
__device__ __forceinline__ uint32_t finite_magnitude(float x) {
    const uint32_t u = __float_as_uint(x) & 0x7FFFFFFFu;
    return u < 0x7F800000u ? u : 0u;
}
// The scale byte for a largest magnitude 1.m * 2^(E - 127): 448 = 1.75 * 2^8.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    const int b = (int)(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return b < 0 ? 0u : (uint32_t)b;
}
__device__ __forceinline__ float scale_of(uint32_t b) { return __uint_as_float(max(b << 23, 0x00400000u)); }
// 2^(127 - b); bytes above 247 come from no float.
__device__ __forceinline__ float unscale_of(uint32_t b) { return __uint_as_float(b < 254u ? (254u - b) << 23 : 0x00400000u); }

// Two values to two codes, the first in the low byte; inf * 0 makes an infinity NaN, the conversion alone would make it 448.
__device__ __forceinline__ uint32_t encode2(float x0, float x1, float unscale) {
    const f32x2 x = pair(x0, x1);
    float y0, y1;
    split(fma2(x, pair(0.f, 0.f), mul2(x, pair(unscale, unscale))), y0, y1);
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(y1), "f"(y0));
    return r;
}
__device__ __forceinline__ uint32_t encode1(float x, float unscale) { return encode2(x, 0.f, unscale) & 0xFFu; }

// Two codes (the low 16 bits) to their values without the scale.
__device__ __forceinline__ void decode2(uint32_t codes, float& x0, float& x1) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)codes));
    asm("{.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;}" : "=f"(x0), "=f"(x1) : "r"(h));
}
__device__ __forceinline__ float decode1(uint32_t code) {
    float x, y;
    decode2(code & 0xFFu, x, y);
    return x;
}

// VE codes to or from one word of VE bytes (1, 4 or 8).
template <int VE> struct CodeWord { using type = uint2; };
template <> struct CodeWord<4> { using type = uint32_t; };
template <> struct CodeWord<1> { using type = uint8_t; };

template <int VE> __device__ __forceinline__ typename CodeWord<VE>::type encode(const float (&x)[VE], float unscale) {
    if constexpr (VE == 1) {
        return (uint8_t)encode1(x[0], unscale);
    } else if constexpr (VE == 4) {
        return encode2(x[0], x[1], unscale) | encode2(x[2], x[3], unscale) << 16;
    } else {
        return make_uint2(encode2(x[0], x[1], unscale) | encode2(x[2], x[3], unscale) << 16, encode2(x[4], x[5], unscale) | encode2(x[6], x[7], unscale) << 16);
    }
}
template <int VE> __device__ __forceinline__ void decode(typename CodeWord<VE>::type w, float (&x)[VE]) {
    if constexpr (VE == 1) {
        x[0] = decode1(w);
    } else if constexpr (VE == 4) {
        decode2(w, x[0], x[1]);
        decode2(w >> 16, x[2], x[3]);
    } else {
        decode2(w.x, x[0], x[1]);
        decode2(w.x >> 16, x[2], x[3]);
        decode2(w.y, x[4], x[5]);
        decode2(w.y >> 16, x[6], x[7]);
    }
}

}  // namespace gs
