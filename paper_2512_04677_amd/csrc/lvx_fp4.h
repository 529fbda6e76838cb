// 4-bit values (E2M1: sign, two exponent bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6) as the gfx950 conversions and matrix instructions take them.
#pragma once
#include "lvx_internal.h"

typedef __attribute__((__vector_size__(8 * sizeof(int)))) int i32x8_t;

#define LVX_FP4_GROUP 32          // consecutive channels that share an E8M0 scale
#define LVX_FP4_MIN_EXPONENT -120 // smallest scale written: every decoded magnitude stays a normal bf16 number

// An E8M0 byte as the fp32 number whose exponent the conversions use: 255 becomes the pattern of infinity, which they take as NaN, as the format does.
__device__ __forceinline__ float lvx_e8m0_f32(uint32_t byte) { return __uint_as_float(byte << 23); }

// Smallest e with amax <= 7 * 2^e as a byte: up to 7 the top level 6 is off by no more than half a step of the levels below it (4, 6), and a larger
// scale would coarsen every other element.  Non-finite amax: 255.
__device__ __forceinline__ uint32_t lvx_fp4_group_byte(uint32_t amax_bits) {
    const int ex = (int)(amax_bits >> 23);
    if (ex == 255) return 255;
    const int byte = ex - 2 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)(byte > 127 + LVX_FP4_MIN_EXPONENT ? byte : 127 + LVX_FP4_MIN_EXPONENT);
}

// Eight codes (element i in bits 4i .. 4i + 3) times the scale: exact in bf16.
__device__ __forceinline__ bf16x8_t lvx_fp4x8_bf16(uint32_t w, float scale) {
    bf16x8_t r;
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    r[0] = a[0], r[1] = a[1], r[2] = b[0], r[3] = b[1], r[4] = c[0], r[5] = c[1], r[6] = d[0], r[7] = d[1];
    return r;
}

// Eight bf16 (two to a word) -> eight codes of x / scale, nearest, ties to the even code, saturating at 6.
__device__ __forceinline__ uint32_t lvx_bf16x8_fp4(uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3, float scale) {
    uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0, *reinterpret_cast<bf16x2_t *>(&x0), scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, *reinterpret_cast<bf16x2_t *>(&x1), scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, *reinterpret_cast<bf16x2_t *>(&x2), scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, *reinterpret_cast<bf16x2_t *>(&x3), scale, 3);
}

// Larger magnitude of the two bf16 of a word and of m (all as bits of fp32 magnitudes, which order like the numbers; a NaN is above infinity and stays).
__device__ __forceinline__ uint32_t lvx_amax_bf16x2(uint32_t m, uint32_t x) {
    const uint32_t lo = (x & 0x7fffu) << 16, hi = x & 0x7fff0000u;
    m = m > lo ? m : lo;
    return m > hi ? m : hi;
}
