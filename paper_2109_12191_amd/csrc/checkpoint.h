// Device helpers of the 8-bit activation checkpoints (format: include/dp_privatise.h, dp_checkpoint_write), shared by the kernels
// that write them and those that contract from them.  gfx950 only.
#pragma once

#include "values.h"

namespace dp {

constexpr int CK_BLOCK = 32;                     // features of a token that share a scale
constexpr int CK_LOW = -100, CK_HIGH = 119;      // exponents of scales: every value is a normal bf16 number, 448 * 2^119 is finite
inline int ck_pitch(int features) { return (features + CK_BLOCK - 1) / CK_BLOCK * CK_BLOCK; }

__device__ __forceinline__ float pow2_of(int biased) { return __uint_as_float((uint32_t)biased << 23); }

// Four codes times 2^(biased - 127) as bf16, two to a dword.  Exact: a code has four significant bits.
__device__ __forceinline__ uint2 ck_bf16(uint32_t codes, float scale)
{
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true)));
}

}  // namespace dp
