// Pages chosen for the queries of a (sequence, KV head) by their mean keys:
//   score_j = max over the rows of q . k_mean_j.
#include <cstdint>
#include <cuda_runtime.h>

#include "cache_choose.cuh"

namespace evisel {
namespace {

constexpr int kScoreThreads = 256;
constexpr int kChooseThreads = 1024;

// A warp per page, a lane per D / 32 channels.
template <class T, int D>
__global__ void __launch_bounds__(kScoreThreads) cache_score_kernel(const __grid_constant__ CacheSelectLaunch L) {
  constexpr int E = D / 32;
  const int h = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 31;
  const int page = blockIdx.x * (kScoreThreads / 32) + (threadIdx.x >> 5);
  const int n = (cache_len(L.c, b, h, L.status) + L.c.page - 1) >> L.c.log_page;
  if (page >= n) return;
  const int64_t id = cache_page(L.c, b, h, page, L.status);
  auto load = [&](const uint16_t* p, float (&x)[E]) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(p + lane * E);
#pragma unroll
    for (int e = 0; e < E / 2; ++e) {
      const uint32_t y = __ldg(w + e);
      x[2 * e] = T::lo(y), x[2 * e + 1] = T::hi(y);
    }
  };
  float k[E];
  load(static_cast<const uint16_t*>(L.c.k_mean) + (id * L.c.hkv + h) * D, k);
  const int drafted = drafted_tokens(L.d, b);
  float top = -INFINITY;
  for (int t = 0; t < drafted; ++t)
    for (int g = 0; g < L.d.gq; ++g) {
      float q[E], x = 0.f;
      load(static_cast<const uint16_t*>(L.d.q) + b * L.d.qs[0] + t * L.d.qs[1] + (h * L.d.gq + g) * L.d.qs[2], q);
#pragma unroll
      for (int e = 0; e < E; ++e) x = fmaf(q[e], k[e], x);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
      top = fmaxf(top, x);
    }
  if (lane == 0) L.scores[(static_cast<int64_t>(b) * L.c.hkv + h) * L.c.max_pages + page] = top;
}

__global__ void __launch_bounds__(kChooseThreads) cache_select_kernel(const __grid_constant__ CacheSelectLaunch L) {
  __shared__ ChooseScratch sc;
  const int b = blockIdx.x / L.c.hkv, h = blockIdx.x % L.c.hkv;
  const int len = cache_len(L.c, b, h, L.status), n = (len + L.c.page - 1) >> L.c.log_page;
  const int count = min(n, L.n_select);
  const bool all = n <= L.n_select;
  const int sink = all ? count : L.sink, recent = all ? 0 : L.recent;
  const float* score = L.scores + (static_cast<int64_t>(b) * L.c.hkv + h) * L.c.max_pages;
  const int64_t at = (static_cast<int64_t>(b) * L.c.hkv + h) * L.n_select;
  auto put = [&](int rank, int page) {
    L.pages[at + rank] = page;
    L.sel_table[at + rank] = cache_page(L.c, b, h, page, L.status);
  };
  for (int i = threadIdx.x; i < sink; i += kChooseThreads) put(i, i);
  for (int i = threadIdx.x; i < recent; i += kChooseThreads) put(count - recent + i, n - recent + i);
  for (int i = count + threadIdx.x; i < L.n_select; i += kChooseThreads) L.pages[at + i] = L.sel_table[at + i] = -1;
  choose_top(sink, n - recent, count - sink - recent, [&](int i) { return order_key(__ldg(score + i)); }, sc,
             [&](int rank, int i) { put(sink + rank, i); });
  if (threadIdx.x == 0)
    L.sel_lens[b * L.c.hkv + h] = count > 0 ? (count - 1) * L.c.page + (len - (n - 1) * L.c.page) : 0;
}

template <class T, int D>
cudaError_t launch_d(const CacheSelectLaunch& L, cudaStream_t stream) {
  constexpr int W = kScoreThreads / 32;
  cache_score_kernel<T, D><<<dim3((L.c.max_pages + W - 1) / W, L.c.hkv, L.c.batch), kScoreThreads, 0, stream>>>(L);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  cache_select_kernel<<<L.c.batch * L.c.hkv, kChooseThreads, 0, stream>>>(L);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_cache_select(const CacheSelectLaunch& L, cudaStream_t stream) {
  if (L.c.dtype == 0) return L.c.head_dim == 128 ? launch_d<BF16, 128>(L, stream) : launch_d<BF16, 64>(L, stream);
  return L.c.head_dim == 128 ? launch_d<FP16, 128>(L, stream) : launch_d<FP16, 64>(L, stream);
}

}  // namespace evisel
