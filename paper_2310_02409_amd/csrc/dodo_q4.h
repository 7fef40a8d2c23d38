// Nugget caches in 4 bits: what the kernels that write and read them share (the format is described in dodo.h).
#pragma once
#include "dodo_common.h"

namespace dodo {

constexpr int kBlockQ4 = 32;          // channels that share a scale
constexpr uint32_t kScaleBadQ4 = 255;  // scale byte of a block with a NaN or an infinity
constexpr int kLeastExpQ4 = -125;     // exponents of a scale: no value but 0 is below 2^-126, the least normal number,
constexpr int kMostExpQ4 = 125;       // and none overflows (6 * 2^125; with 126 a 3.9 would round to 4 * 2^126)

// The scale 2^(byte - 127) as fp32 (bytes 2 .. 252; for 255 an infinity, with which the conversions below give NaN for every code).
__device__ __forceinline__ float scale_q4(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight channels (the codes of 4 bytes, the lowest first) as four pairs of bf16.  The conversion multiplies by the scale's power of
// two: exact, e2m1 has two bits of mantissa.
__device__ __forceinline__ uint4 unpack8_bf16(uint32_t codes, float scale) {
  uint4 v;
  v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
  v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  return v;
}

// The scale bytes of a row and head (BLOCKS of them, aligned to as many), the first one lowest; and whether one is kScaleBadQ4.
template <int BLOCKS>
__device__ __forceinline__ uint32_t row_scales_q4(const uint8_t* scales, int64_t row_head) {
  static_assert(BLOCKS == 2 || BLOCKS == 4, "64 or 128 channels");
  if (BLOCKS == 2) return reinterpret_cast<const uint16_t*>(scales)[row_head];
  return reinterpret_cast<const uint32_t*>(scales)[row_head];
}
__device__ __forceinline__ bool any_bad_q4(uint32_t scales) {
  static_assert(kScaleBadQ4 == 255, "all bits of a byte");
  return ((~scales - 0x01010101u) & scales & 0x80808080u) != 0;  // a byte of ~scales is 0
}

// dodo_unpack_nuggets_q4; `for_attention` (d_h 64 or 128): a K/V row and head with a bad block in K is all zeros there in that block, and
// NaN in all channels of V.
int unpack_q4(const uint8_t* Kc, const uint8_t* Ks, const uint8_t* Vc, const uint8_t* Vs, int64_t rows, int32_t d_h, int dtype,
              bool for_attention, void* Kn, void* Vn, void* stream);

}  // namespace dodo
