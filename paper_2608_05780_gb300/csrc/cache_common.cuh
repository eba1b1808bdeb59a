// Device helpers of the paged-cache kernels: checked lengths and page ids, the
// 16-bit types, mma.sync and ldmatrix, and the even split of ragged work.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "cache_internal.h"
#include "cache_split.h"
#include "sm103_ptx.cuh"

namespace evisel {

__device__ __forceinline__ void record_bounds(int* status) { atomicExch(status, kStatusBounds); }

// Tokens of (sequence, head), clamped to what a table row can hold.
__device__ __forceinline__ int cache_len(const CacheView& c, int b, int h, int* status) {
  const int n = __ldg(c.lens + b * c.ls[0] + h * c.ls[1]);
  const int64_t room = static_cast<int64_t>(c.max_pages) << c.log_page;
  if (n >= 0 && n <= room) return n;
  record_bounds(status);
  return n < 0 ? 0 : static_cast<int>(room);
}

// Page id of logical page j (j < max_pages) to write to: -1 where the table holds none of the pool.
__device__ __forceinline__ int cache_page_to_write(const CacheView& c, int b, int h, int j, int* status) {
  const int id = __ldg(c.table + b * c.ts[0] + h * c.ts[1] + j);
  if (static_cast<unsigned>(id) < static_cast<unsigned>(c.n_pages)) return id;
  record_bounds(status);
  return -1;
}

// The same to read from: a page of the pool whatever the table holds.
__device__ __forceinline__ int cache_page(const CacheView& c, int b, int h, int j, int* status) {
  return max(0, cache_page_to_write(c, b, h, j, status));
}

__device__ __forceinline__ int drafted_tokens(const DraftView& d, int b) {
  if (!d.drafted) return d.tokens;
  const int n = __ldg(d.drafted + b);
  return n < 0 ? 0 : n < d.tokens ? n : d.tokens;
}

// ---------------------------------------------------------------- 16-bit types
// kHeadroom: log2 units by which a softmax's reference exponent stands below the
// running maximum where weights are rounded to this type. fp16 ends at 2^-24: without
// it weights below 2^-25 of the maximum were lost from O but not from the row sum
// (16,000 keys at 2^-26: 2^-12 of the values). With 7, and a maximum that is up to
// 2^8 stale, weights stay below 2^15 and are kept down to 2^-32.
struct BF16 {
  static constexpr float kHeadroom = 0.f;
  static constexpr uint32_t kFormat = 1;         // operand format of a kind::f16 tcgen05.mma
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return ptx::pack_bf16x2(lo, hi); }
  static __device__ __forceinline__ float lo(uint32_t x) { return __uint_as_float(x << 16); }
  static __device__ __forceinline__ float hi(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
};
struct FP16 {
  static constexpr float kHeadroom = 7.f;
  static constexpr uint32_t kFormat = 0;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
  }
  static __device__ __forceinline__ float lo(uint32_t x) {
    return __half2float(__ushort_as_half(static_cast<unsigned short>(x & 0xffffu)));
  }
  static __device__ __forceinline__ float hi(uint32_t x) {
    return __half2float(__ushort_as_half(static_cast<unsigned short>(x >> 16)));
  }
};

// Eight 16-bit values to fp32.
template <class T>
__device__ __forceinline__ void unpack8(const uint4& w, float (&f)[8]) {
  f[0] = T::lo(w.x), f[1] = T::hi(w.x), f[2] = T::lo(w.y), f[3] = T::hi(w.y);
  f[4] = T::lo(w.z), f[5] = T::hi(w.z), f[6] = T::lo(w.w), f[7] = T::hi(w.w);
}

namespace ptx {

// Programmatic dependent launch: grid_wait() returns when the kernels before this
// one in the stream have ended and their writes are visible; a kernel calls
// grid_launch_next() after it, so that whatever may start early finds everything
// before the kernel it follows done.
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_launch_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// 4-D tiled load whose token, head and page (or sequence) coordinates stand at the places that
// `perm` names: two bits each for the coordinate (1..3) of token, head and page.
__device__ __forceinline__ void tma_load_page(uint32_t dst, const CUtensorMap* map, uint32_t bar, int perm, int c0,
                                              int token, int head, int page, uint64_t cache_hint) {
  const int pt = perm & 3, ph = (perm >> 2) & 3;
  const int c1 = pt == 1 ? token : ph == 1 ? head : page;
  const int c2 = pt == 2 ? token : ph == 2 ? head : page;
  const int c3 = pt == 3 ? token : ph == 3 ? head : page;
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%2, %3, %4, %5}], [%6], %7;" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar), "l"(cache_hint)
      : "memory");
}

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldmatrix4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}

// c (16 x 8, fp32) += a (16 x 16) b (16 x 8)
template <class T>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (T::kFormat == 1)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

}  // namespace ptx

// ---------------------------------------------------------------- even split of ragged work
// Sequences (or (sequence, head) pairs, where each has its length) are entries of
// `mult` problems each. A problem holds `lead` units for its fill and its join,
// then one per key_tile keys; nothing where it has no key. Every thread of the block calls; `mem` holds 2 + 32 ints.
struct Split {
  int total;        // units of all entries
  int entry;        // the entry that was looked for ...
  int first;        // ... and its first unit
};

struct UnitCount {
  const CacheView& c;
  int key_tile, lead, mult;
  int* status;
  bool per_head;
  __device__ __forceinline__ UnitCount(const CacheView& c_, int key_tile_, int lead_, int row_tiles, int* status_)
      : c(c_), key_tile(key_tile_), lead(lead_), mult(0), status(status_), per_head(c_.ls[1] != 0) {
    mult = per_head ? row_tiles : row_tiles * c.hkv;
  }
  __device__ __forceinline__ int entries() const { return per_head ? c.batch * c.hkv : c.batch; }
  __device__ __forceinline__ int tiles(int e) const {
    const int len = per_head ? cache_len(c, e / c.hkv, e % c.hkv, status) : cache_len(c, e, 0, status);
    return (len + key_tile - 1) / key_tile;
  }
  __device__ __forceinline__ int units(int tiles) const { return tiles > 0 ? tiles + lead : 0; }   // of a problem
};

// Exclusive prefix over the block of one int per thread; `total` gets the sum. Two barriers.
__device__ __forceinline__ int block_prefix(int x, int* warp_sums, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = (blockDim.x + 31) >> 5;
  int inc = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int w = 0; w < n_warps; ++w) {
    const int s = warp_sums[w];
    if (w < warp) before += s;
    total += s;
  }
  __syncthreads();
  return before + inc - x;
}

constexpr int kWarpEntries = 256;                // up to so many entries every warp adds up by itself

// The entry that holds unit `at(total)`. Every thread of the block calls and gets it.
template <class At>
__device__ __forceinline__ Split split_find_unit(const UnitCount& u, int* mem, At at) {
  const int n = u.entries();
  Split s;
  if (n <= kWarpEntries) {
    // Without a barrier: a block's first loads wait for nothing but the lengths.
    const int lane = threadIdx.x & 31;
    if (n <= 32) {                               // (little code: it is fetched cold)
      const int m = lane < n ? u.units(u.tiles(lane)) * u.mult : 0;
      int inc = m;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      s.total = __shfl_sync(0xffffffffu, inc, 31);
      const int want = at(s.total);
      const uint32_t hit = __ballot_sync(0xffffffffu, want >= inc - m && want < inc);
      s.entry = hit ? __ffs(hit) - 1 : 0;
      s.first = __shfl_sync(0xffffffffu, inc - m, s.entry);
      return s;
    }
    // Each lane adds up a run of entries, one scan joins the lanes, and the lane
    // that holds the unit looks through its run.
    const int per = (n + 31) / 32, e0 = lane * per;
    int m[kWarpEntries / 32], sum = 0;
#pragma unroll
    for (int c = 0; c < kWarpEntries / 32; ++c) {
      m[c] = c < per && e0 + c < n ? u.units(u.tiles(e0 + c)) * u.mult : 0;
      sum += m[c];
    }
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    s.total = __shfl_sync(0xffffffffu, inc, 31);
    const int want = at(s.total);
    int first = inc - sum, entry = e0;
    bool past = true;                            // the entries so far all end before it
    const uint32_t hit = __ballot_sync(0xffffffffu, want >= first && want < inc);
#pragma unroll
    for (int c = 0; c < kWarpEntries / 32; ++c) {
      past = past && want >= first + m[c];
      if (past) first += m[c], ++entry;
    }
    const int src = hit ? __ffs(hit) - 1 : 0;
    s.entry = hit ? __shfl_sync(0xffffffffu, entry, src) : 0;
    s.first = hit ? __shfl_sync(0xffffffffu, first, src) : 0;
    return s;
  }
  const int per = (n + static_cast<int>(blockDim.x) - 1) / static_cast<int>(blockDim.x);
  const int e0 = min(n, static_cast<int>(threadIdx.x) * per), e1 = min(n, e0 + per);
  int sum = 0;
  for (int e = e0; e < e1; ++e) sum += u.units(u.tiles(e)) * u.mult;
  int first = block_prefix(sum, mem + 2, s.total);
  const int want = at(s.total);
  if (threadIdx.x == 0) mem[0] = mem[1] = 0;
  __syncthreads();
  if (want >= first && want < first + sum)
    for (int e = e0; e < e1; ++e) {
      const int m = u.units(u.tiles(e)) * u.mult;
      if (want < first + m) {
        mem[0] = e;
        mem[1] = first;
        break;
      }
      first += m;
    }
  __syncthreads();
  s.entry = mem[0];
  s.first = mem[1];
  return s;
}

// The first unit of entry `want`, likewise.
__device__ __forceinline__ Split split_find_entry(const UnitCount& u, int* mem, int want) {
  const int n = u.entries();
  Split s;
  s.entry = want;
  if (n <= kWarpEntries) {
    const int lane = threadIdx.x & 31;
    int all = 0, before = 0;
#pragma unroll
    for (int c = 0; c < kWarpEntries / 32; ++c) {
      const int e = c * 32 + lane, m = e < n ? u.units(u.tiles(e)) * u.mult : 0;
      all += m;
      before += e < want ? m : 0;
    }
    s.total = __reduce_add_sync(0xffffffffu, all);
    s.first = __reduce_add_sync(0xffffffffu, before);
    return s;
  }
  const int per = (n + static_cast<int>(blockDim.x) - 1) / static_cast<int>(blockDim.x);
  const int e0 = min(n, static_cast<int>(threadIdx.x) * per), e1 = min(n, e0 + per);
  int sum = 0, before = 0;
  for (int e = e0; e < e1; ++e) {
    const int m = u.units(u.tiles(e)) * u.mult;
    if (e < want) before += m;
    sum += m;
  }
  const int first = block_prefix(sum, mem + 2, s.total);
  if (want >= e0 && want < e1) mem[1] = first + before;
  __syncthreads();
  s.first = mem[1];
  return s;
}

// ---------------------------------------------------------------- launch
// Launches a kernel that begins with grid_wait() (or waits before it reads what
// the kernel before it writes).
template <class... Params>
cudaError_t launch_after(void (*kern)(Params...), dim3 grid, unsigned threads, size_t smem, cudaStream_t stream,
                         const Params&... params) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, params...);
}

// The same in clusters of `cluster` CTAs, one per problem.
template <class Launch>
cudaError_t launch_clusters(void (*kern)(Launch), const Launch& L, int problems, unsigned threads, int cluster,
                            cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(problems * cluster);
  cfg.blockDim = dim3(threads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, L);
}

}  // namespace evisel
