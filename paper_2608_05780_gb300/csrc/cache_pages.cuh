// One page of a cache filled from a source of tokens, with its mean key.
#pragma once

#include "cache_common.cuh"

namespace evisel {

constexpr int kPageThreads = 256;
// Tokens of a thread in flight, blocks per SM: an append of 65,664 tokens took 49 us with four tokens and
// as many blocks as their registers leave, 43 with two and five.
constexpr int kAtOnce = 2, kPageBlocks = 5;

// Writes the page's slots at positions [src.first(), src.end()) and, with
// `mean`, the mean of all its keys before src.end() (the older ones read back
// from the page). A block of kPageThreads threads per (page, head, sequence); D / 8
// threads share a token, 16 bytes of it each.
template <class T, int D, class Source>
__device__ __forceinline__ void fill_page(const CacheView& c, void* k_out, void* v_out, void* mean, int b, int h, int page,
                                          const Source& src, int* status) {
  constexpr int LANES = D / 8, GROUPS = kPageThreads / LANES;
  __shared__ float sums[GROUPS][D];
  const int p0 = page << c.log_page, p1 = min(p0 + c.page, src.end());
  if (p1 <= p0 || p1 <= src.first()) return;     // (the whole block)
  const int64_t id = cache_page_to_write(c, b, h, page, status);
  if (id < 0) return;                            // (the whole block: any other page has its own tokens)
  uint16_t* k = static_cast<uint16_t*>(k_out) + id * c.ks[0] + h * c.ks[1];
  uint16_t* v = static_cast<uint16_t*>(v_out) + id * c.vs[0] + h * c.vs[1];
  const int x = threadIdx.x % LANES, grp = threadIdx.x / LANES;
  float sum[8] = {};
  // kAtOnce tokens a thread at a time: their places, then all loads, then all stores.
  for (int base = p0 + grp; base < p1; base += kAtOnce * GROUPS) {
    const uint4 *ks[kAtOnce], *vs[kAtOnce];
    uint4 key[kAtOnce], value[kAtOnce];
    bool in[kAtOnce], fresh[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int pos = base + i * GROUPS;
      fresh[i] = pos < p1 && pos >= src.first();
      in[i] = fresh[i] || (pos < p1 && mean);    // an older token is read for the mean only
      ks[i] = vs[i] = reinterpret_cast<const uint4*>(k + (pos - p0) * c.ks[2]);
      if (fresh[i]) src.rows(pos, ks[i], vs[i]);
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      key[i] = in[i] ? ks[i][x] : make_uint4(0, 0, 0, 0);
      if (fresh[i]) value[i] = vs[i][x];
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int slot = base + i * GROUPS - p0;
      if (fresh[i]) {
        reinterpret_cast<uint4*>(k + slot * c.ks[2])[x] = key[i];
        reinterpret_cast<uint4*>(v + slot * c.vs[2])[x] = value[i];
      }
      float f[8];
      unpack8<T>(key[i], f);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += in[i] ? f[e] : 0.f;
    }
  }
  if (!mean) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[grp][x * 8 + e] = sum[e];
  __syncthreads();
  const float n = static_cast<float>(p1 - p0);
  uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(mean) + (id * c.hkv + h) * D);
  for (int i = threadIdx.x; i < D / 2; i += kPageThreads) {
    float lo = 0.f, hi = 0.f;
    for (int g = 0; g < GROUPS; ++g) {
      lo += sums[g][2 * i];
      hi += sums[g][2 * i + 1];
    }
    dst[i] = T::pack(lo / n, hi / n);
  }
}

}  // namespace evisel
