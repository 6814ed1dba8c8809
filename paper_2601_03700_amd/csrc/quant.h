// Weights in 4 bits: OCP e2m1 codes (0, 1/2, 1, 3/2, 2, 3, 4, 6 and a sign) with one
// power of two 2^E, stored as 127 + E, for every 32 of a row.  A value has at most two
// significant bits, so it is exact in bf16: products with it are those of the bf16
// matrix that adept_quant_unpack gives.
//
// A matrix [n][k] is held in blocks of 16 rows and 128 of K, those of 16 rows next to
// each other, zeros behind n and k.  A block's 1024 bytes are the 16 bytes that each
// lane of a wave needs as the first operand of four v_mfma_f32_16x16x32_bf16: lane l
// has row l % 16, its dword h the eight k = 32 h + 8 (l / 16) .. + 7, the first in the
// lowest four bits.  A block's 64 scale bytes are four for each row.
#pragma once

#include "common.h"

namespace adept {

constexpr int kQuantK = 128, kQuantRows = 16;   // of a block
constexpr int kQuantBlock = 1024, kQuantScales = 64;   // bytes of its codes, of its scales
constexpr int kQuantScaleMin = 127 - 100, kQuantScaleMax = 127 + 100;
constexpr uint8_t kQuantScaleNan = 255;
inline int64_t quant_blocks(int n, int k) {
  return (int64_t)ceil_div(n, kQuantRows) * ceil_div(k, kQuantK);
}

// Eight codes times the scale in the low byte of `byte`.  The scale byte 255 makes them NaN.
__device__ __forceinline__ bf16x8_t quant_expand(uint32_t codes, uint32_t byte) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const float s = __uint_as_float((byte & 255u) << 23);
  u32x4 w;
  w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0));
  w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1));
  w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2));
  w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3));
  return __builtin_bit_cast(bf16x8_t, w);
}

}  // namespace adept
