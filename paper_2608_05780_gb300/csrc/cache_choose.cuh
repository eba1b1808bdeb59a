// Choice of the highest of many scores by one cluster of CTAs: a radix select on
// their order keys over shared-memory histograms (read across the cluster),
// then their positions in ascending order.
#pragma once

#include "cache_common.cuh"

namespace evisel {

namespace ptx {
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The int at shared address `addr` of CTA `rank` of the cluster.
__device__ __forceinline__ int ld_cluster(uint32_t addr, uint32_t rank) {
  uint32_t a;
  int v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
}  // namespace ptx

// Ascending with the float (-0 equal to 0), NaN lowest.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (isnan(x)) return 0u;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct ChooseMem {
  int hist[4][256];                 // per pass: the keys of this CTA by digit
  int tot[256];
  int digit, left, done;
  int above[32], tie[32];           // per warp
  int sum[2];                       // this CTA's keys above the boundary, and on it
};

// A CTA's part [a, b) of [lo, hi): whole groups of 32 in order of rank.
struct ChoosePart {
  int a, b, chunk;
  __device__ __forceinline__ ChoosePart(int lo, int hi, int rank, int size) {
    chunk = (max(hi - lo, 0) + 32 * size - 1) / (32 * size) * 32;
    a = min(hi, lo + rank * chunk);
    b = min(hi, a + chunk);
  }
};

// The sum over the cluster of the int at `p`, read from every CTA at once.
__device__ __forceinline__ int sum_cluster(const int* p, int size) {
  int x[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) x[r] = r < size ? ptx::ld_cluster(ptx::smem_addr(p), r) : 0;
  return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
}

// The `want` highest of key(i), lo <= i < hi (0 <= want <= hi - lo; ties: the
// lower i): emit(rank, i) for each, ranks ascending with i. Every thread of every
// CTA of the cluster calls, with the same lo, hi and want; key(i) is asked for
// the i of the CTA's own ChoosePart only. The last cluster barrier is the
// caller's: no CTA may leave before the others have read its sums. THREADS: the
// block's; rank, size: the CTA's place in the cluster (0, 1: the block by itself).
// meanwhile(): what the caller does while the keys are on their way.
// A warp owns a run of the part; a thread keeps up to ITEMS keys of its run in
// registers, so that a part of up to ITEMS * THREADS scores is read once.
template <int THREADS, int ITEMS, class Key, class Emit, class Meanwhile>
__device__ __forceinline__ void choose_top(int lo, int hi, int want, Key key, ChooseMem& m, Emit emit, int rank, int size,
                                           Meanwhile meanwhile) {
  if (want <= 0) {
    meanwhile();
    return;
  }
  const ChoosePart part(lo, hi, rank, size);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int run = ((part.b - part.a + THREADS - 1) / THREADS) * 32;
  const int wa = min(part.b, part.a + warp * run), wb = min(part.b, wa + run);
  const bool held = run <= 32 * ITEMS;
  uint32_t keys[ITEMS];
  if (held && wa < wb) {                         // (past the run its last key again: no branch between the loads)
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) keys[it] = key(min(wa + 32 * it + lane, wb - 1));
  }
  meanwhile();
  // f(key, i, whether i is of the run) for the run's keys in order, 32 at a time.
  auto each = [&](auto f) {
    if (held) {
#pragma unroll
      for (int it = 0; it < ITEMS; ++it)
        if (wa + 32 * it < wb) f(keys[it], wa + 32 * it + lane, wa + 32 * it + lane < wb);
    } else {
#pragma unroll 4
      for (int i = wa + lane; i - lane < wb; i += 32) f(i < wb ? key(i) : 0u, i, i < wb);
    }
  };
  uint32_t prefix = 0, mask = 0;                 // the boundary's digits so far
  int left = want;                               // to take among the keys with that prefix
  for (int i = threadIdx.x; i < 4 * 256; i += THREADS) m.hist[i >> 8][i & 255] = 0;
  __syncthreads();
  for (int pass = 0; pass < 4; ++pass) {
    const int shift = 24 - 8 * pass;
    each([&](uint32_t k, int, bool in) {
      if (in && (k & mask) == prefix) atomicAdd(&m.hist[pass][(k >> shift) & 255u], 1);
    });
    if (size > 1) ptx::cluster_sync();
    else __syncthreads();
    if (size > 1 && threadIdx.x < 256) m.tot[threadIdx.x] = sum_cluster(&m.hist[pass][threadIdx.x], size);
    if (size > 1) __syncthreads();
    if (warp == 0) {
      // Digits from the highest: a lane holds eight, the one where the sum reaches `left` walks them.
      const int* tot = size > 1 ? m.tot : m.hist[pass];
      int x[8], sum = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += x[e] = tot[255 - 8 * lane - e];
      int inc = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      int rest = left - (inc - sum);
      if (rest > 0 && rest <= sum) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (rest > 0 && rest <= x[e]) {
            m.digit = 255 - 8 * lane - e;
            m.left = rest;
            m.done = rest == x[e];               // all keys with this prefix are taken: no digit below it matters
          }
          rest -= x[e];
        }
      }
    }
    __syncthreads();
    prefix |= static_cast<uint32_t>(m.digit) << shift;
    mask |= 255u << shift;
    left = m.left;
    if (m.done) break;
  }
  // Keys above the boundary, and the first `left` on it: counted per run, then placed.
  int above = 0, tie = 0;
  each([&](uint32_t k, int, bool in) {
    above += __popc(__ballot_sync(0xffffffffu, in && (k & mask) > prefix));
    tie += __popc(__ballot_sync(0xffffffffu, in && (k & mask) == prefix));
  });
  if (lane == 0) {
    m.above[warp] = above;
    m.tie[warp] = tie;
  }
  __syncthreads();
  if (warp == 0) {
    const int xa = lane < THREADS / 32 ? m.above[lane] : 0, xt = lane < THREADS / 32 ? m.tie[lane] : 0;
    int ia = xa, it = xt;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int ya = __shfl_up_sync(0xffffffffu, ia, o), yt = __shfl_up_sync(0xffffffffu, it, o);
      if (lane >= o) {
        ia += ya;
        it += yt;
      }
    }
    m.above[lane] = ia - xa;
    m.tie[lane] = it - xt;
    if (lane == 31) {
      m.sum[0] = ia;
      m.sum[1] = it;
    }
  }
  if (size > 1) ptx::cluster_sync();
  else __syncthreads();
  // Before this warp's run: the runs before it, and the CTAs before this one (a lane each).
  int na = 0, nt = 0;
  if (size > 1) {
    if (lane < rank) {
      na = ptx::ld_cluster(ptx::smem_addr(&m.sum[0]), lane);
      nt = ptx::ld_cluster(ptx::smem_addr(&m.sum[1]), lane);
    }
    na = __reduce_add_sync(0xffffffffu, na);
    nt = __reduce_add_sync(0xffffffffu, nt);
  }
  na += m.above[warp];
  nt += m.tie[warp];
  each([&](uint32_t k, int i, bool in) {
    const bool is_above = in && (k & mask) > prefix, is_tie = in && (k & mask) == prefix;
    const uint32_t ba = __ballot_sync(0xffffffffu, is_above), bt = __ballot_sync(0xffffffffu, is_tie);
    const uint32_t low = (1u << lane) - 1u;
    const int ta = na + __popc(ba & low), tt = nt + __popc(bt & low);
    if (is_above || (is_tie && tt < left)) emit(ta + min(tt, left), i);
    na += __popc(ba);
    nt += __popc(bt);
  });
}

// CTAs per problem: one for work up to `alone`, else as many as stay within one CTA
// per SM (each exchange within a cluster costs about a microsecond whatever its size;
// with more CTAs than SMs the clusters wait for room: 32 problems of 8 took 17.9 us, of 4 6.8).
inline int choose_cluster(int64_t problems, int64_t work, int64_t alone, int n_sm) {
  int c = work > alone ? 8 : 1;
  while (c > 1 && problems * c > n_sm) c /= 2;
  return c;
}

}  // namespace evisel
