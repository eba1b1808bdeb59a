// What the attention kernels over a paged cache share: bounded waits and a
// CTA's walk over its part of the units.
#pragma once

#include "cache_common.cuh"

namespace evisel {

constexpr float kRescaleThreshold = 8.0f;        // log2 units: a running max moves only when it grows by more

__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  const bool ok = ptx::mbar_wait(bar, parity, abort_flag, kWaitTimeoutNs);
  return __all_sync(0xffffffffu, ok);
}

__device__ __forceinline__ void record_timeout(volatile int* abort_flag, int* status) {
  *abort_flag = 1;
  atomicExch(status, kStatusTimeout);
}

// A CTA's part of one problem: key tiles [t0, t1) of a (sequence, KV head, row tile).
struct Segment {
  int b, h, rt, t0, t1, len, problem;
};

// A CTA's segments in order, from unit u on.
struct Walk {
  int u, end, entry, first;
  __device__ __forceinline__ bool next(const CacheView& c, int row_tiles, const UnitCount& uc, Segment& s, int* status) {
    for (;;) {
      if (u >= end) return false;
      int tiles = uc.tiles(entry), n = uc.units(tiles);
      while (u >= first + n * uc.mult) {
        first += n * uc.mult;
        tiles = uc.tiles(++entry);
        n = uc.units(tiles);
      }
      const int inner = (u - first) / n, from = (u - first) % n, to = min(n, from + (end - u));
      u += to - from;
      s.t0 = max(0, from - uc.lead);
      s.t1 = max(0, to - uc.lead);
      if (s.t0 == s.t1) continue;                // a problem's lead alone: its keys are the next CTA's
      s.b = uc.per_head ? entry / c.hkv : entry;
      s.h = uc.per_head ? entry % c.hkv : inner / row_tiles;
      s.rt = inner % row_tiles;
      s.len = cache_len(c, s.b, s.h, status);
      s.problem = (s.b * c.hkv + s.h) * row_tiles + s.rt;
      return true;
    }
  }
};

}  // namespace evisel
