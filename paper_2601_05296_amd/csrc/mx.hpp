// mx.hpp -- microscaled 4-bit floating point (the OCP Microscaling format MXFP4) on gfx950.
//
// 32 consecutive values share one scale byte s, standing for 2^(s - 127) (255: NaN), and
// each value is a 4-bit e2m1 code: sign, then 0, 0.5, 1, 1.5, 2, 3, 4, 6. Value 2i of a
// block is the low half of its byte i, value 2i + 1 the high half.
#pragma once

#include "common.hpp"

namespace moe {
namespace mx {

constexpr int BLOCK = 32;

// The scale byte of a block whose largest magnitude has these float32 bits (sign clear):
// 2^(floor(log2(largest)) - 2), so that the largest lands in [4, 8) and no scale is lost to
// the codes' two exponent bits; never below 2^-127. Infinity or NaN: 255.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    const uint32_t e = top >> 23;
    return e == 255u ? 255u : e < 2u ? 0u : e - 2u;
}

// A scale byte as float32, exact (0 is the subnormal 2^-127, 255 a NaN).
__device__ __forceinline__ float scale_value(uint32_t byte) {
    return __uint_as_float(byte == 0u ? 0x00400000u : byte == 255u ? 0x7fc00000u : byte << 23);
}

// Eight values over `scale` as codes, to nearest, ties to the even code, saturating at 6
// (v_cvt_scalef32_pk_fp4_f32; checked against the definition over every finite bfloat16 and
// float32 values around each border, scales 2^-126 to 2^120).
__device__ __forceinline__ uint32_t encode8(const float (&v)[8], float scale) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
    return c;
}

// Eight codes times `scale` as bfloat16 (exact inside bfloat16's range; all 256 pairs of
// codes checked, scales 2^-127 to 2^127).
__device__ __forceinline__ uint4 decode8(uint32_t c, float scale) {
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    uint4 v;
    v.x = __builtin_bit_cast(uint32_t, (bf2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0));
    v.y = __builtin_bit_cast(uint32_t, (bf2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1));
    v.z = __builtin_bit_cast(uint32_t, (bf2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2));
    v.w = __builtin_bit_cast(uint32_t, (bf2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3));
    return v;
}

}  // namespace mx
}  // namespace moe
