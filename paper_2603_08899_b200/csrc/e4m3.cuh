// E4M3 (OCP 8-bit floating point) conversions and the scale rule of block-scaled caches.
#pragma once

#include "common.cuh"

namespace confu {

// four floats -> four codes (a in the lowest byte), round to nearest even, saturating at +-448, NaN stays NaN
__device__ __forceinline__ uint32_t e4m3_pack4(float a, float b, float c, float d)
{
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
        "mov.b32 %0, {lo, hi};\n\t}"
        : "=r"(r)
        : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}

// four codes -> two pairs of f16 (every E4M3 value is an f16 value)
__device__ __forceinline__ void e4m3_to_f16x4(uint32_t codes, uint32_t& lo, uint32_t& hi)
{
    asm("{\n\t.reg .b16 a, b;\n\t"
        "mov.b32 {a, b}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, a;\n\t"
        "cvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(codes));
}

__device__ __forceinline__ void f16x2_to_f32(uint32_t v, float& a, float& b)
{
    asm("{\n\t.reg .b16 x, y;\n\t"
        "mov.b32 {x, y}, %2;\n\t"
        "cvt.f32.f16 %0, x;\n\t"
        "cvt.f32.f16 %1, y;\n\t}"
        : "=f"(a), "=f"(b)
        : "r"(v));
}

__device__ __forceinline__ void e4m3_to_f32x4(uint32_t codes, float (&x)[4])
{
    uint32_t lo, hi;
    e4m3_to_f16x4(codes, lo, hi);
    f16x2_to_f32(lo, x[0], x[1]);
    f16x2_to_f32(hi, x[2], x[3]);
}

// Or-ed together for any number of words: bits of 0x80808080 are set where one of the codes is not a number (0x7f, 0xff).
__device__ __forceinline__ uint32_t e4m3_nan_trace(uint32_t codes) { return (codes & 0x7f7f7f7fu) + 0x01010101u; }
constexpr uint32_t kNanTrace = 0x80808080u;
// 0xff in the place of every code that is not a number
__device__ __forceinline__ uint32_t e4m3_nan4(uint32_t codes) { return __vcmpeq4(codes & 0x7f7f7f7fu, 0x7f7f7f7fu); }

// The smallest power of two 2^e, e >= -100, with amax <= 448 * 2^e (448 = 0.875 * 2^9), for a finite amax >= 0.  A power of two: encoding
// an entry again for a block whose scale has grown then only drops bits below the smallest E4M3 step, it never rounds
// a rounded value a second time, and scale times code is exact.
constexpr int kLeastScaleExp = -100;
__device__ __forceinline__ float e4m3_block_scale(float amax)
{
    const uint32_t bits = __float_as_uint(amax);
    // amax = 1.f * 2^(E - 127) = (1.f / 2) * 2^(E - 126); more than 0.875 where 1.f > 1.75.  (0 and subnormals: below the least.)
    const int e = (int)(bits >> 23) - 126 - 9 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return __uint_as_float((uint32_t)(max(e, kLeastScaleExp) + 127) << 23);
}

}  // namespace confu
