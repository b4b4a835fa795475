// The 4-bit cache's format, as the hardware converts it.
//
// 32 consecutive elements of a head share the power of two 2^(s - 127), s a byte;
// an element is a sign, two bits of exponent and one of fraction:
//   code & 7    0   1    2   3    4   5   6   7
//   level       0  0.5   1  1.5   2   3   4   6
// A level is exact in bf16 at every scale that appends write (two significant bits;
// under s of 253 and 254 the larger levels are infinite), so that attention multiplies
// what the cache stands for, with no further rounding.
#pragma once

#include "attn_device.h"
#include "fp4_launch.h"

namespace ssn {

constexpr int kNanScale = 255;         // reads back as 32 NaN

// The scale 2^(s - 127) as the conversions take it (its exponent bits).
__device__ __forceinline__ float fp4_scale(uint32_t s) { return __uint_as_float(s << 23); }

// The scale byte of a group whose largest magnitude has the bits `top` (of the
// absolute values as whole numbers, which puts NaN above infinity): the smallest
// e with max < 7 2^e, so that the largest rounds to 6 at most (7 is as far from 6
// as from 8, and 8 is the even one).  With max = 1.f 2^(E - 127) that is E - 129,
// or E - 128 from 1.75 on.  -126 <= e <= 125: below, a group holds less than its
// 2 bits; above, 6 2^e would be infinite, and what is larger becomes 6 2^125.
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t top) {
  if (top >= 0x7F800000u) return kNanScale;
  const int s = (int)(top >> 23) - 2 + ((top & 0x7FFFFFu) >= 0x600000u);
  return (uint32_t)clampi(s, 1, 252);
}
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Two elements to a byte of codes, nearest level, ties to the even code.
template <int BYTE>
__device__ __forceinline__ uint32_t fp4_pack(uint32_t into, float a, float b, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(into, a, b, scale, BYTE);
}
// The two elements of byte BYTE, as bf16 in a dword and in float32.
template <int BYTE>
__device__ __forceinline__ uint32_t fp4_bf16x2(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, BYTE));
}
template <int BYTE>
__device__ __forceinline__ f32x2 fp4_f32x2(uint32_t codes, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, BYTE);
}
// The eight elements of a dword as bf16.
__device__ __forceinline__ u32x4 fp4_bf16x8(uint32_t codes, float scale) {
  return u32x4{fp4_bf16x2<0>(codes, scale), fp4_bf16x2<1>(codes, scale), fp4_bf16x2<2>(codes, scale),
               fp4_bf16x2<3>(codes, scale)};
}

// The largest of v over LANES (4 or 8) neighbouring lanes, in each of them.
template <int LANES>
__device__ __forceinline__ uint32_t lanes_umax(uint32_t v) {
  v = umax(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));     // lane ^ 1
  v = umax(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));     // lane ^ 2
  // of 8 lanes the one at the other end: both fours hold theirs everywhere
  if constexpr (LANES == 8) v = umax(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true));
  return v;
}
// Codes of a lane's E elements (8 or 4) of a group that 32 / E neighbouring lanes
// hold, and the group's scale byte.
template <int E>
__device__ __forceinline__ uint32_t fp4_quantise(const float (&v)[E], uint32_t& s) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) top = umax(top, abs_bits(v[e]));
  s = fp4_scale_byte(lanes_umax<kFp4Group / E>(top));
  const float scale = fp4_scale(s);
  uint32_t codes = fp4_pack<1>(fp4_pack<0>(0, v[0], v[1], scale), v[2], v[3], scale);
  if constexpr (E == 8) codes = fp4_pack<3>(fp4_pack<2>(codes, v[4], v[5], scale), v[6], v[7], scale);
  return s == kNanScale ? 0 : codes;
}

}  // namespace ssn
