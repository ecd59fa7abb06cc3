// K/V rows in 4 bits.  32 neighbouring elements of a row share a scale 2^(b - 127), b a byte (255: not a number), and
// each is a code of 4 bits: a sign and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 (two bits of exponent, one of fraction).  A byte
// holds two codes, the even element's in its low half.  Rows of a head follow each other: d/2 bytes of codes each; the
// scales, d/32 bytes a row, stand behind the codes of all heads.  A row of 128 bf16 elements takes 68 bytes
// instead of 256.  The values have two significant bits, so bf16 holds each of them exactly down to its least exponent.
#pragma once

#include "fc_common.hpp"

typedef __bf16 fc_bf16x2_t __attribute__((ext_vector_type(2)));
typedef float fc_f32x4_t __attribute__((ext_vector_type(4)));

// Eight codes and their scale's byte -> eight bf16 values.  The conversion takes the scale's exponent from a float's, and its
// exponent of all ones gives NaN.
__device__ __forceinline__ u32x4_native fc_kv4_to_bf16(uint32_t codes, uint32_t scale_byte) {
    const float s = __uint_as_float(scale_byte << 23);
    u32x4_native r;
    r.x = __builtin_bit_cast(uint32_t, (fc_bf16x2_t)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0));
    r.y = __builtin_bit_cast(uint32_t, (fc_bf16x2_t)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1));
    r.z = __builtin_bit_cast(uint32_t, (fc_bf16x2_t)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2));
    r.w = __builtin_bit_cast(uint32_t, (fc_bf16x2_t)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3));
    return r;
}

// Four codes and their scale's byte -> four floats
__device__ __forceinline__ fc_f32x4_t fc_kv4_to_f32(uint32_t codes, uint32_t scale_byte) {
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    const float s = __uint_as_float(scale_byte << 23);
    const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 1);
    return fc_f32x4_t{a.x, a.y, b.x, b.y};
}
