// Choice of the highest of many scores by one block: a radix select on their
// order keys, then their positions in ascending order.
#pragma once

#include "cache_common.cuh"

namespace evisel {

// Ascending with the float (-0 equal to 0), NaN lowest.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (isnan(x)) return 0u;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct ChooseScratch {
  int hist[256];
  int digit, left;
  int sums[34];
};

// The `want` highest of key(i), lo <= i < hi (0 <= want <= hi - lo; ties: the
// lower i): emit(rank, i) for each, ranks ascending with i. The whole block calls.
template <class Key, class Emit>
__device__ __forceinline__ void choose_top(int lo, int hi, int want, Key key, ChooseScratch& sc, Emit emit) {
  if (want <= 0) return;
  const int n = hi - lo, threads = blockDim.x;
  uint32_t prefix = 0, mask = 0;                 // the boundary key's digits so far
  int left = want;                               // to take among the keys with that prefix
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += threads) sc.hist[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += threads) {
      const uint32_t k = key(lo + i);
      if ((k & mask) == prefix) atomicAdd(&sc.hist[(k >> shift) & 255u], 1);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      int d = 255, rest = left;
      while (d > 0 && sc.hist[d] < rest) rest -= sc.hist[d--];
      sc.digit = d;
      sc.left = rest;
    }
    __syncthreads();
    prefix |= static_cast<uint32_t>(sc.digit) << shift;
    mask |= 255u << shift;
    left = sc.left;
  }
  // Keys above the boundary key, and the first `left` equal to it.
  int rank = 0, equal = 0;
  for (int base = 0; base < n; base += threads) {
    const int i = base + static_cast<int>(threadIdx.x);
    const uint32_t k = i < n ? key(lo + i) : 0u;
    const bool above = i < n && k > prefix, tie = i < n && k == prefix;
    int total, total_eq;
    const int eq = equal + block_prefix(tie, sc.sums, total_eq);
    const bool take = above || (tie && eq < left);
    const int at = rank + block_prefix(take, sc.sums, total);
    if (take) emit(at, lo + i);
    rank += total;
    equal += total_eq;
  }
}

}  // namespace evisel
