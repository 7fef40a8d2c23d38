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

// First position p of list[0 .. n) (ascending) with list[p] >= value, n if there is none.  Called by whole wavefronts: 64 places
// are looked at in each step, so a list of 4096 takes two memory latencies.
__device__ __forceinline__ int lower_bound_wave(const int32_t* __restrict__ list, int n, int value) {
  int lo = 0, hi = n;  // the answer is in [lo, hi]
  while (hi > lo) {
    const int step = (hi - lo + kWave - 1) / kWave;
    const int at = lo + lane_id() * step;
    const uint64_t below = __ballot(at < hi && list[min(at, hi - 1)] < value);  // a run of lanes from 0 on
    const int cnt = __popcll(below);
    if (cnt == 0) return lo;
    const int last = lo + (cnt - 1) * step;  // the last place looked at that is below
    hi = min(hi, last + step);
    lo = last + 1;
  }
  return lo;
}

}  // namespace dodo
