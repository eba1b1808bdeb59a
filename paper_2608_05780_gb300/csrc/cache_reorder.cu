// The beams that go on: tables and lengths by parent, the pages in progress of
// further children copied, other states by row, all in one launch: a block per sequence and head
// (or several heads, of up to 32 KB of a page: 512 sequences of eight heads of 64 with pages of 16 take 8.1 us, 10.8 head by
// head) and per 16 KB of a state's row. Each block finds out by itself whose pages its sequence takes (64 parents are two
// registers of a warp), rather than wait for another kernel. Small calls are its dependent loads (parents, lengths, table, page):
// 3.9 us for four beams; 128 beams with 135 KB of states each take 9.0, 70% of a plain copy's rate.
#include "cache_common.cuh"
#include "decode_internal.h"

namespace evisel {
namespace {

constexpr int kThreads = 256;
constexpr int kVectors = kStateBytes / 16 / kThreads;   // of a state row's block, per thread

// Parent of slot j of a group, itself where none is named.
__device__ __forceinline__ int parent_of(const ReorderLaunch& L, int64_t group, int j) {
  const int p = __ldg(L.parent + group * L.beams + j);
  if (p >= L.beams) record_bounds(L.status);
  return p < 0 || p >= L.beams ? j : p;
}

// The slot whose own pages slot `child` takes, by one warp. A bit of a 64-bit mask per slot: `have` those with a
// child; the first child of a parent keeps its pages, the e-th other one takes the e-th slot's that has none.
__device__ __forceinline__ int donor_of(const ReorderLaunch& L, int64_t group, int child, int& parent) {
  const int lane = threadIdx.x & 31;
  const bool in0 = lane < L.beams, in1 = lane + 32 < L.beams;
  const int p0 = in0 ? parent_of(L, group, lane) : -1, p1 = in1 ? parent_of(L, group, lane + 32) : -1;
  const unsigned same0 = __match_any_sync(0xffffffffu, p0), same1 = __match_any_sync(0xffffffffu, p1);
  const uint64_t bit0 = in0 ? uint64_t(1) << p0 : 0, bit1 = in1 ? uint64_t(1) << p1 : 0;
  const uint64_t have0 = __reduce_or_sync(0xffffffffu, static_cast<unsigned>(bit0)) |
                         static_cast<uint64_t>(__reduce_or_sync(0xffffffffu, static_cast<unsigned>(bit0 >> 32))) << 32;
  const uint64_t have = have0 | __reduce_or_sync(0xffffffffu, static_cast<unsigned>(bit1)) |
                        static_cast<uint64_t>(__reduce_or_sync(0xffffffffu, static_cast<unsigned>(bit1 >> 32))) << 32;
  const bool later0 = in0 && __ffs(same0) - 1 != lane;
  const bool later1 = in1 && (__ffs(same1) - 1 != lane || (have0 & bit1) != 0);
  const uint64_t later = __ballot_sync(0xffffffffu, later0) | static_cast<uint64_t>(__ballot_sync(0xffffffffu, later1)) << 32;
  const int pa = __shfl_sync(0xffffffffu, p0, child & 31), pb = __shfl_sync(0xffffffffu, p1, child & 31);
  parent = child < 32 ? pa : pb;
  if (!(later >> child & 1)) return parent;
  const uint64_t slots = L.beams == 64 ? ~uint64_t(0) : (uint64_t(1) << L.beams) - 1;
  uint64_t free = slots & ~have;                 // as many as there are later children
  for (int skip = __popcll(later & ((uint64_t(1) << child) - 1)); skip > 0; --skip) free &= free - 1;
  return __ffsll(static_cast<long long>(free)) - 1;
}

// The first `tokens` of a page, `heads` of its heads from h0 on; 1 << log_lanes threads to a row.
__device__ __forceinline__ void copy_rows(const void* pool, void* out, const int64_t (&s)[3], int from, int to, int h0, int heads,
                                          int tokens, int log_lanes) {
  const uint16_t* src = static_cast<const uint16_t*>(pool) + from * s[0];
  uint16_t* dst = static_cast<uint16_t*>(out) + to * s[0];
  for (int i = threadIdx.x; i < heads * tokens << log_lanes; i += kThreads) {
    const int row = i >> log_lanes, x = i - (row << log_lanes), h = heads == 1 ? 0 : row / tokens, t = row - h * tokens;
    const int64_t at = (h0 + h) * s[1] + t * s[2];
    reinterpret_cast<uint4*>(dst + at)[x] = reinterpret_cast<const uint4*>(src + at)[x];
  }
}

__global__ void __launch_bounds__(kThreads) cache_reorder_kernel(const __grid_constant__ ReorderLaunch L) {
  ptx::grid_wait();
  ptx::grid_launch_next();
  const CacheView& c = L.c;
  if (static_cast<int>(blockIdx.x) < L.first_block[0]) {          // a sequence's head, or some
    const int shares = (c.hkv + L.heads - 1) / L.heads, seq = blockIdx.x / shares, h = (blockIdx.x - seq * shares) * L.heads;
    const int heads = min(L.heads, c.hkv - h), log_lanes = c.head_dim == 64 ? 3 : 4, group = seq / L.beams, first = group * L.beams;
    int p;
    const int d = donor_of(L, group, seq - first, p) + first;
    p += first;
    const int len = cache_len(c, p, 0, L.status), full = len >> c.log_page, rest = len & (c.page - 1);
    if (h == 0) {
      if (threadIdx.x == 0) L.lens_out[seq] = len;
      const int32_t *tp = c.table + p * c.ts[0], *td = c.table + d * c.ts[0];
      for (int m = threadIdx.x; m < c.max_pages; m += kThreads)
        L.table_out[static_cast<int64_t>(seq) * c.max_pages + m] = __ldg((m < full ? tp : td) + m);
    }
    if (d == p) return;
    if (cache_len(c, d, 0, L.status) >> c.log_page > full) {      // its pages so far may be another's too
      record_bounds(L.status);
      return;
    }
    if (rest == 0) return;
    const int from = cache_page_to_write(c, p, 0, full, L.status), to = cache_page_to_write(c, d, 0, full, L.status);
    if (from < 0 || to < 0) return;
    copy_rows(c.k, L.k, c.ks, from, to, h, heads, rest, log_lanes);
    copy_rows(c.v, L.v, c.vs, from, to, h, heads, rest, log_lanes);
    if (L.k_mean) {
      const uint4* m = static_cast<const uint4*>(L.k_mean) + ((static_cast<int64_t>(from) * c.hkv + h) << log_lanes);
      uint4* out = static_cast<uint4*>(L.k_mean) + ((static_cast<int64_t>(to) * c.hkv + h) << log_lanes);
      for (int i = threadIdx.x; i < heads << log_lanes; i += kThreads) out[i] = m[i];
    }
    return;
  }
  int s = 0;
  while (s + 1 < L.n_states && static_cast<int>(blockIdx.x) >= L.first_block[s + 1]) ++s;
  const int at = blockIdx.x - L.first_block[s], seq = at / L.chunks[s], group = seq / L.beams;
  const int64_t bytes = L.row_bytes[s], begin = static_cast<int64_t>(at - seq * L.chunks[s]) * kStateBytes;
  const int p = group * L.beams + parent_of(L, group, seq - group * L.beams);
  const char* in = L.in[s] + p * bytes + begin;
  char* out = L.out[s] + seq * bytes + begin;
  const int n = static_cast<int>(min(static_cast<int64_t>(kStateBytes), bytes - begin));
  if (((reinterpret_cast<uintptr_t>(in) | reinterpret_cast<uintptr_t>(out) | n) & 15) == 0) {
    uint4 x[kVectors];
#pragma unroll
    for (int i = 0; i < kVectors; ++i)
      if ((threadIdx.x + i * kThreads) * 16 < n) x[i] = reinterpret_cast<const uint4*>(in)[threadIdx.x + i * kThreads];
#pragma unroll
    for (int i = 0; i < kVectors; ++i)
      if ((threadIdx.x + i * kThreads) * 16 < n) reinterpret_cast<uint4*>(out)[threadIdx.x + i * kThreads] = x[i];
  } else if (((reinterpret_cast<uintptr_t>(in) | reinterpret_cast<uintptr_t>(out) | n) & 3) == 0) {
    for (int i = threadIdx.x; i < n / 4; i += kThreads) reinterpret_cast<uint32_t*>(out)[i] = reinterpret_cast<const uint32_t*>(in)[i];
  } else {
    for (int i = threadIdx.x; i < n; i += kThreads) out[i] = in[i];
  }
}

}  // namespace

cudaError_t launch_reorder(const ReorderLaunch& L, cudaStream_t stream) {
  return launch_after(cache_reorder_kernel, dim3(static_cast<unsigned>(L.first_block[L.n_states])), kThreads, 0, stream, L);
}

}  // namespace evisel
