// mx_common.h -- device helpers of the block-scaled kernels.
//
// E2M1 codes become bf16 values (and back) in the gfx950 conversion instructions, two
// elements at a time, the block's scale included.  Over all 256 code pairs and 256 scale
// bytes they give the exact value, subnormal results and the NaN of byte 255 among them,
// and over all finite bf16 inputs the nearest code, ties to even, saturated.
#pragma once

#include "gemm_common.h"
#include "mx.h"

namespace gemm {

typedef unsigned u32x4_any_mx __attribute__((ext_vector_type(4), aligned(1)));
typedef unsigned u32x2_any_mx __attribute__((ext_vector_type(2), aligned(1)));
typedef unsigned u32_any_mx __attribute__((aligned(1)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// The scale operand of the conversions for scale byte e: they use its exponent field.
__device__ __forceinline__ float mx4_scale(uint32_t e) { return __builtin_bit_cast(float, e << 23); }

// Eight 4-bit codes (element i in bits 4 i) to eight bf16 values, two to a dword.
__device__ __forceinline__ u32x4_t mx4_to_bf16(uint32_t codes, float scale) {
    return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
}

// 2^(e - 127) as fp32; NaN for e = 255.
__device__ __forceinline__ float mx_scale(uint32_t e) {
    return __builtin_bit_cast(float, e == 0u ? 0x00400000u : e == 255u ? 0x7fc00000u : e << 23);
}

// Four int8 codes (element i in byte i) times a scale to four bf16 values.  A code has seven
// significant bits and the scale one, so the product is a bf16 number and its upper half
// all of it.
__device__ __forceinline__ u32x2_t mx8_to_bf16(uint32_t codes, float scale) {
    const float f0 = float(int8_t(codes)) * scale, f1 = float(int8_t(codes >> 8)) * scale;
    const float f2 = float(int8_t(codes >> 16)) * scale, f3 = float(int8_t(codes >> 24)) * scale;
    return u32x2_t{perm(__builtin_bit_cast(uint32_t, f1), __builtin_bit_cast(uint32_t, f0), 0x07060302u),
                   perm(__builtin_bit_cast(uint32_t, f3), __builtin_bit_cast(uint32_t, f2), 0x07060302u)};
}

__device__ __forceinline__ float bf16_to_f32(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }

}  // namespace gemm
