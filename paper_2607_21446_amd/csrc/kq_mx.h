// Blocks of 32 values that share an E8M0 scale: E2M1 (MXFP4) and E4M3 (MXFP8)
// elements of a cache and a weight, to and from 16 and 32 bits.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kq {

namespace {

typedef uint32_t u32x2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Two values rounded to bf16 (nearest, ties to even).
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    bf16x2 v;
    v[0] = (__bf16)a;
    v[1] = (__bf16)b;
    return __builtin_bit_cast(uint32_t, v);
}

// The scale operand of the conversions: the float with exponent field s (its mantissa is ignored, 0 is 2^-127).
__device__ __forceinline__ float mx_scale(uint32_t s) { return __uint_as_float(s << 23); }

// E8M0 byte of a block whose largest magnitude is amax (finite): its exponent field minus the element's largest.
template <int MOST>
__device__ __forceinline__ uint32_t mx_byte(float amax) {
    const uint32_t e = __float_as_uint(amax) >> 23;
    return e > MOST ? e - MOST : 0u;
}

// Two values 2 I, 2 I + 1 of a word of codes, as bf16.  The scale's subnormals do not come up: a block that has one
// holds values below 2^-124.
template <int I>
__device__ __forceinline__ uint32_t e2m1_pair(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, I));
}
template <int I>
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, I));
}

// Eight values as codes.
__device__ __forceinline__ uint32_t e2m1_codes(const float (&v)[8], float scale) {
    uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
}
// (The conversion's own saturation is not relied on: 448 is the largest code's value.)
__device__ __forceinline__ u32x2v e4m3_codes(const float (&v)[8], float scale) {
    typedef int16_t s16x2 __attribute__((ext_vector_type(2)));
    // 448 scale in 32 bits: a block's own scale is at most 2^(254 - 8 - 127), and 0 stands for 2^-127
    const float top = 448.0f * (scale == 0.0f ? __uint_as_float(0x00400000u) : scale);
    u32x2v c;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __builtin_amdgcn_fmed3f(v[4 * k + i], -top, top);
        s16x2 w = {0, 0};
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, f[0], f[1], scale, false);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, f[2], f[3], scale, true);
        c[k] = __builtin_bit_cast(uint32_t, w);
    }
    return c;
}

}  // namespace

}  // namespace kq
