// Parts that the attention kernels for a few query vectors share (plain and 4-bit caches): products of NV x NV blocks, and the
// online softmax of 32 keys.
#pragma once
#include "dodo_attn.h"

namespace dodo {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) short shortx4;
typedef __attribute__((ext_vector_type(8))) float floatx8;
typedef __attribute__((ext_vector_type(16))) float floatx16;
typedef __attribute__((address_space(3))) void lds_void;

constexpr float kNegInf = -__builtin_inff();

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }  // exp2(-inf) = 0
constexpr int vmcnt_imm(int n) { return 0x0f70 | (n & 15) | ((n >> 4) << 14); }         // s_waitcnt vmcnt(n) only

typedef __attribute__((ext_vector_type(4))) float floatx4;
template <int NV>
struct Mfma;  // accumulator of NV x NV floats; a product is 16 (NV = 32) or 32 (NV = 16) deep
template <>
struct Mfma<32> {
  typedef floatx16 Acc;
  static constexpr int kRegs = 16;
  __device__ static __forceinline__ Acc mul(const bf16x8& a, const bf16x8& b, const Acc& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mfma<16> {
  typedef floatx4 Acc;
  static constexpr int kRegs = 4;
  __device__ static __forceinline__ Acc mul(const bf16x8& a, const bf16x8& b, const Acc& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};

// Largest / sum of x over the lanes of a query vector (the lanes of equal index modulo NV).
template <int NV>
__device__ __forceinline__ float vector_max(float x) {
  float a, b;
  if (NV == 16) {
    lane_pair<16>(x, a, b);
    x = fmaxf(a, b);
  }
  lane_pair<32>(x, a, b);
  return fmaxf(a, b);
}
template <int NV>
__device__ __forceinline__ float vector_sum(float x) {
  float a, b;
  if (NV == 16) {
    lane_pair<16>(x, a, b);
    x = a + b;
  }
  lane_pair<32>(x, a, b);
  return a + b;
}

// Online-softmax update for one 32-key tile.  acc holds the raw S^T accumulators: register v <-> key 8 (v / 4) + 4 g + v % 4
// (NV = 32, g = lane / 32) or 16 (v / 4) + 4 g + v % 4 (NV = 16, g = lane / 16).  MASK: keys at or beyond `limit` are masked.
// Returns P^T as the MFMA B operands (NV = 32: k-step t covers keys 16t .. 16t+15) in PARTS parts: the weights' upper 8 bits of
// mantissa, and what they lack, in bf16 again.  With two they count with 16 bits, and O's error is that of its own rounding to
// bf16 (2-norm against 64 bits 1.66e-3; 2.1e-3 to 2.3e-3 with weights rounded to bf16); the matrix pipe, which is idle three
// quarters of the time here, does twice the work for V (64 sequences of 667 rows, 64 heads over 8: 32.4 -> 33.3 us).  With three they
// are whole, as in the split-K kernel: calls that come here only to be faster than there have these (with two, one value of O in 250
// rounded to another neighbour than the 64-bit result does, with three one in 6000, as there; 6 sequences of 357 rows, 64 heads over 8
// 6.6 -> 6.7 us, 14 of 457 9.2 -> 9.6).  No part of a weight is negative, nor zero unless the weight is: with an
// infinity in V their products are that infinity.  A lower part is `least` at least, or the weight itself, which then counts twice: with
// the default that shows where the keys of weight 1 have a V below 2^-100, which 4-bit blocks may hold and their kernel asks for less.
// The exponent offset m_run of a vector is moved (and its sum and output accumulators rescaled) only when the tile's
// maximum exceeds it by more than kSlack: the result does not depend on the offset, the weights stay below
// 2^kSlack, and after the first tiles of a vector the output accumulators are hardly ever touched again (the rescale is
// a wavefront-uniform branch: taken if any vector of the wavefront moves).
constexpr float kSlack = 8.f;
template <bool MASK, int NV, int CB, int REGS, int PARTS>
__device__ __forceinline__ void softmax_tile32(float (&acc)[REGS], int limit, int g, float scale_log2e, float& m_run,
                                               float& l_run, typename Mfma<NV>::Acc (&acc_o)[CB], bf16x8 (&pf)[PARTS][REGS / 8],
                                               float least = 1e-30f) {
  float tmax = kNegInf;
#pragma unroll
  for (int v = 0; v < REGS; ++v) {
    float s = acc[v] * scale_log2e;
    if (MASK) {
      const int key = (NV == 32 ? 8 : 16) * (v >> 2) + 4 * g + (v & 3);
      s = (key < limit) ? s : kNegInf;
    }
    acc[v] = s;
    tmax = fmaxf(tmax, s);
  }
  tmax = vector_max<NV>(tmax);                // all lanes of a vector decide alike
  const bool move = tmax > m_run + kSlack;  // (m_run = -inf: any finite maximum moves it)
  if (__any(move)) {
    const float m_new = move ? tmax : m_run;
    const float alpha = exp2_hw(m_run - ((m_new == kNegInf) ? 0.f : m_new));  // 1 where nothing moves, 0 from -inf
    l_run *= alpha;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int v = 0; v < Mfma<NV>::kRegs; ++v) acc_o[cb][v] *= alpha;
    m_run = m_new;
  }
  const float m_use = (m_run == kNegInf) ? 0.f : m_run;
  float psum = 0.f;
#pragma unroll
  for (int half = 0; half < REGS / 8; ++half) {
    floatx8 low;
    uint32_t high[PARTS - 1][4];
#pragma unroll
    for (int v = 0; v < 8; v += 2) {
      const float p0 = exp2_hw(acc[8 * half + v] - m_use), p1 = exp2_hw(acc[8 * half + v + 1] - m_use);
      psum += p0;
      psum += p1;
      float r0 = p0, r1 = p1;
#pragma unroll
      for (int part = 0; part < PARTS - 1; ++part) {
        const uint32_t b0 = __float_as_uint(r0), b1 = __float_as_uint(r1);
        high[part][v / 2] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);  // the upper halves: rounded towards zero
        r0 = __builtin_amdgcn_fmed3f(r0 - __uint_as_float(b0 & 0xffff0000u), least, p0);
        r1 = __builtin_amdgcn_fmed3f(r1 - __uint_as_float(b1 & 0xffff0000u), least, p1);
      }
      low[v] = r0;
      low[v + 1] = r1;
    }
#pragma unroll
    for (int part = 0; part < PARTS - 1; ++part)
      pf[part][half] = __builtin_bit_cast(bf16x8, make_uint4(high[part][0], high[part][1], high[part][2], high[part][3]));
    pf[PARTS - 1][half] = __builtin_convertvector(low, bf16x8);  // hardware round-to-nearest-even pack
  }
  l_run += psum;
}

}  // namespace dodo
