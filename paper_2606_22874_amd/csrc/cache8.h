// An 8-bit cache (gfx950): e4m3 codes, and a power of two for every 16 tokens of a head.
//
// An element is code 2^(b - 127), b the byte of its 16 tokens.  With four significant bits
// and a power of two it is a BF16 number as it stands (FP16 within that type's range), so
// that one conversion of two codes, scale included, gives what the matrix instructions
// take, and attention over such a cache is that over a 16-bit one of the same values.
#pragma once

#include "paged_core.h"

namespace spot {
namespace paged {

// The scale of a byte, as the conversions take it: they read its exponent (0: 2^-127,
// 255: NaN).
__device__ __forceinline__ float scale8(uint32_t byte) {
  return __builtin_bit_cast(float, byte << 23);
}

// Four codes times a scale, as two pairs of the element type.
__device__ __forceinline__ u32x2 wide4(Bf16, uint32_t codes, float scale) {
  return u32x2{__builtin_bit_cast(uint32_t,
                                  __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false)),
               __builtin_bit_cast(uint32_t,
                                  __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true))};
}
__device__ __forceinline__ u32x2 wide4(Fp16, uint32_t codes, float scale) {
  return u32x2{__builtin_bit_cast(uint32_t,
                                  __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, false)),
               __builtin_bit_cast(uint32_t,
                                  __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, true))};
}
template <class T>
__device__ __forceinline__ u32x4 wide8(uint32_t a, uint32_t b, float sa, float sb) {
  const u32x2 x = wide4(T(), a, sa), y = wide4(T(), b, sb);
  return u32x4{x[0], x[1], y[0], y[1]};
}

// Whether one of four codes is NaN.
__device__ __forceinline__ bool nan4(uint32_t codes) {
  return (((codes & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0u;
}
// Scales from here on take the largest code (448) past the element type's numbers.
template <class T>
__device__ __forceinline__ bool far8(uint32_t byte);
template <>
__device__ __forceinline__ bool far8<Bf16>(uint32_t byte) { return byte >= 127 + 120; }
template <>
__device__ __forceinline__ bool far8<Fp16>(uint32_t byte) { return byte >= 127 + 8; }

}  // namespace paged
}  // namespace spot
