// Lookups in the packed index lists, shared by the kernels that follow a nugget to its token and back.
#pragma once
#include "dodo_common.h"

namespace dodo {

// The sequence b with cu[b] <= row < cu[b + 1], or -1 for a row from cu[B] on; row >= 0.  Up to 64 sequences: one boundary per lane
// and a ballot, so that the lookup is a single memory latency; beyond, a binary search.  Called by whole wavefronts.
__device__ __forceinline__ int sequence_of(const int32_t* __restrict__ cu, int B, int64_t row) {
  if (B <= kWave) {
    const int lane = lane_id();
    const int bound = cu[min(lane + 1, B)];
    const uint64_t above = __ballot(lane < B && bound > row);
    return above == 0 ? -1 : __ffsll(static_cast<long long>(above)) - 1;
  }
  if (row >= cu[B]) return -1;
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= row) lo = mid; else hi = mid;
  }
  return lo;
}

// The token (of all sequences') that cache row `row` holds, or -1 behind the last sequence's; nugget_idx[row] exists.  Up to 64
// sequences: everything is fetched at once.  Called by whole wavefronts.
__device__ __forceinline__ int64_t token_of(const int32_t* __restrict__ cu_seqlens, const int32_t* __restrict__ cu_nuggets,
                                            const int32_t* __restrict__ nugget_idx, int B, int64_t row) {
  if (B <= kWave) {
    const int lane = lane_id();
    const int bound = cu_nuggets[min(lane + 1, B)], start = cu_seqlens[min(lane, B)], idx = nugget_idx[row];
    const uint64_t above = __ballot(lane < B && bound > row);
    if (above == 0) return -1;
    return static_cast<int64_t>(__builtin_amdgcn_readlane(start, __ffsll(static_cast<long long>(above)) - 1)) + idx;
  }
  const int b = sequence_of(cu_nuggets, B, row);
  return b < 0 ? -1 : static_cast<int64_t>(cu_seqlens[b]) + nugget_idx[row];
}

// The sequences' token and nugget ranges, found by token.  Up to 64 sequences: a sequence per lane, all of it fetched at once.
struct SequenceLookup {
  const int32_t *cu_seqlens, *cu_nuggets;
  int B, s0_l, s1_l, k0_l, k1_l;
  __device__ __forceinline__ SequenceLookup(const int32_t* cu_seqlens_, const int32_t* cu_nuggets_, int B_)
      : cu_seqlens(cu_seqlens_), cu_nuggets(cu_nuggets_), B(B_) {
    if (B <= kWave) {
      const int lane = lane_id();
      s0_l = cu_seqlens[min(lane, B)];
      s1_l = cu_seqlens[min(lane + 1, B)];
      k0_l = cu_nuggets[min(lane, B)];
      k1_l = cu_nuggets[min(lane + 1, B)];
    }
  }
  // Ranges [s0, s1) of tokens and [k0, k1) of nuggets of the sequence that token `tok` belongs to; false behind the last one.
  __device__ __forceinline__ bool find(int64_t tok, int& s0, int& s1, int& k0, int& k1) const {
    if (B <= kWave) {
      const uint64_t above = __ballot(lane_id() < B && s1_l > tok);
      if (above == 0) return false;
      const int b = __ffsll(static_cast<long long>(above)) - 1;
      s0 = __builtin_amdgcn_readlane(s0_l, b);
      s1 = __builtin_amdgcn_readlane(s1_l, b);
      k0 = __builtin_amdgcn_readlane(k0_l, b);
      k1 = __builtin_amdgcn_readlane(k1_l, b);
      return true;
    }
    const int b = sequence_of(cu_seqlens, B, tok);
    if (b < 0) return false;
    s0 = cu_seqlens[b];
    s1 = cu_seqlens[b + 1];
    k0 = cu_nuggets[b];
    k1 = cu_nuggets[b + 1];
    return true;
  }
};

// A place p0 <= p in list[0 .. n) (ascending), where p is the first with list[p] >= value (n if there is none), no more than 64 before
// it.  64 places are looked at in each step: one memory latency for a list of up to 4096.
__device__ __forceinline__ int before_lower_bound(const int32_t* __restrict__ list, int n, int value) {
  int lo = 0, hi = n;  // p is in [lo, hi]
  while (hi - lo > kWave) {
    const int step = (hi - lo + kWave - 1) / kWave, at = lo + lane_id() * step;
    const int cnt = __popcll(__ballot(at < hi && list[min(at, hi - 1)] < value));  // a run of lanes from 0 on
    if (cnt == 0) return lo;
    lo += (cnt - 1) * step + 1;  // behind the last place looked at that is below
    hi = min(hi, lo - 1 + step);
  }
  return lo;
}

}  // namespace dodo
