// f8.cuh -- 8-bit floating point (e4m3: four exponent bits, three mantissa bits, largest value
// 448) with a power-of-two scale for each block of 128.
//
// A block's scale is the smallest 2^e >= max |v| / 448 (e >= -126): v / 2^e is exact, so the only
// rounding is the one to e4m3's three mantissa bits, and the largest value lands between 224 and
// 448.  Against a scale of max / 448 itself this gives up at most one of e4m3's 15 binades at the
// small end and saves a rounding of every value and of every product with the scale.  A block of
// zeros has scale 1; one that holds an infinity or a NaN has scale NaN, so that everything
// computed from it is NaN instead of a plausible number.
#pragma once
#include <cstdint>

#include "ptx.cuh"

namespace quan {

constexpr int F8_BLOCK = 128;

// Scale of a block from its largest magnitude, and the factor 1 / scale.
__device__ __forceinline__ float f8_scale(float amax, float& inv) {
    const uint32_t u = __float_as_uint(amax);  // amax >= 0
    int e = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    e = e < -126 ? -126 : e;
    if (u == 0u) e = 0;
    if (u >= 0x7F800000u) {
        inv = 0.0f;
        return __uint_as_float(0x7FC00000u);
    }
    inv = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
    return __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
}

// max(|v|) over values that may be NaN or infinite: the largest bit pattern without its sign
// (NaN above infinity above every number).
__device__ __forceinline__ uint32_t abs_bits(float v) {
    return __float_as_uint(v) & 0x7FFFFFFFu;
}

// Two values to e4m3, nearest even, magnitudes above 448 to 448: `lo` in the low byte.
__device__ __forceinline__ uint32_t f8x2_from_f32(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t f8x4_from_f32(float a, float b, float c, float d) {
    return f8x2_from_f32(a, b) | (f8x2_from_f32(c, d) << 16);
}

// The four e4m3 values of a word, lowest byte first (exact).
__device__ __forceinline__ void f8x4_to_f32(uint32_t w, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(w >> (16 * i))));
        asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\t"
            "cvt.f32.f16 %1, b;\n\t}"
            : "=f"(v[2 * i]), "=f"(v[2 * i + 1])
            : "r"(h));
    }
}

__device__ __forceinline__ float f8_to_f32(uint8_t b) {
    float v[4];
    f8x4_to_f32(b, v);
    return v[0];
}

// ------------------------------------------------------------------ activations

// SiLU z / (1 + e^-z), e^-z = 2^(-z log2 e), with the hardware's approximate 2^x and reciprocal,
// and no cap on the exponent: from z = -87.3 down the divisor passes 2^126, its reciprocal is
// flushed to 0 and the result is -0, where SiLU lies above -2^-119.  (A capped exponent leaves a
// sigmoid that never falls further: -1e20 would give a number far from 0.)  -inf gives NaN, as
// -inf / (1 + inf) does.
__device__ __forceinline__ float f8_silu(float z) {
    return z * rcp_approx_ftz(1.0f + ex2_approx_ftz(z * -1.44269504f));
}

// The epilogue's activation; a NaN stays one (a block without a scale has to show).
__device__ __forceinline__ float f8_act(float z, int act) {
    return act == 1 ? (z < 0.0f ? 0.0f : z) : (act == 2 ? f8_silu(z) : z);
}

}  // namespace quan
