// Eviction: the tokens of a (sequence, KV head) with the most accumulated
// weight, its sinks and its recent ones, compacted into other pages. The copy
// gathers rows of 256 bytes (d = 128): 134 MB, read and written, in 25 us.
#include <cstdint>
#include <cuda_runtime.h>

#include "cache_choose.cuh"
#include "cache_pages.cuh"

namespace evisel {
namespace {

// 512 threads of at most 64 registers: two CTAs fit an SM, so that clusters of
// eight find room in every GPC (of 1,024 one in sixteen waited for the others to
// end: four caches of 65,664 took 33 us, with 512 it is 20). Three or four dependent
// passes over the digits, 1.5 us each, and not the 4 MB of scores are the bound.
constexpr int kChooseThreads = 512;

__global__ void __launch_bounds__(kChooseThreads, 2) cache_evict_choose_kernel(const __grid_constant__ CacheEvictLaunch L) {
  __shared__ ChooseMem mem;
  ptx::grid_wait();
  ptx::grid_launch_next();
  const int rank = static_cast<int>(ptx::cluster_rank()), size = static_cast<int>(ptx::cluster_size());
  const int problem = blockIdx.x / size, b = problem / L.c.hkv, h = problem % L.c.hkv;
  int len = cache_len(L.c, b, h, L.status);
  if (len > L.acc_len) {
    record_bounds(L.status);
    len = static_cast<int>(L.acc_len);
  }
  const int count = min(len, L.budget);
  const bool all = len <= L.budget;
  const int sink = all ? count : L.sink, recent = all ? 0 : L.recent;
  const float* acc = L.acc + static_cast<int64_t>(problem) * L.acc_len;
  int32_t* kept = L.kept + static_cast<int64_t>(problem) * L.budget;
  float* out = L.acc_out + static_cast<int64_t>(problem) * L.acc_out_len;
  auto put = [&](int place, int i) {
    kept[place] = i;
    out[place] = acc[i];
  };
  const int first = rank * kChooseThreads + static_cast<int>(threadIdx.x), step = size * kChooseThreads;
  choose_top<kChooseThreads, 16>(
      sink, len - recent, count - sink - recent, [&](int i) { return order_key(__ldg(acc + i)); }, mem,
      [&](int place, int i) { put(sink + place, i); }, rank, size, [&]() {
        for (int i = first; i < sink; i += step) put(i, i);
        for (int i = first; i < recent; i += step) put(count - recent + i, len - recent + i);
        for (int i = count + first; i < L.budget; i += step) kept[i] = -1;
        for (int64_t i = count + first; i < L.acc_out_len; i += step) out[i] = 0.f;
      });
  if (first == 0) L.out_lens[b * L.out.ls[0] + h * L.out.ls[1]] = count;
  if (size > 1) ptx::cluster_sync();
}

// The source of an evicted cache's page: the kept tokens, in order.
struct KeptTokens {
  const CacheEvictLaunch& L;
  int b, h, count;
  const int32_t* kept;
  __device__ __forceinline__ KeptTokens(const CacheEvictLaunch& L_, int b_, int h_) : L(L_), b(b_), h(h_) {
    count = min(cache_len(L.c, b, h, L.status), L.budget);
    if (count > L.acc_len) count = static_cast<int>(L.acc_len);
    kept = L.kept + (static_cast<int64_t>(b) * L.c.hkv + h) * L.budget;
  }
  __device__ __forceinline__ int first() const { return 0; }             // positions written: [first, end)
  __device__ __forceinline__ int end() const { return count; }
  __device__ __forceinline__ void rows(int pos, const uint4*& k, const uint4*& v) const {
    const int i = __ldg(kept + pos);
    const int64_t id = cache_page(L.c, b, h, i >> L.c.log_page, L.status), slot = i & (L.c.page - 1);
    k = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(L.c.k) + id * L.c.ks[0] + h * L.c.ks[1] + slot * L.c.ks[2]);
    v = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(L.c.v) + id * L.c.vs[0] + h * L.c.vs[1] + slot * L.c.vs[2]);
  }
};

template <class T, int D>
__global__ void __launch_bounds__(kPageThreads, kPageBlocks) cache_evict_copy_kernel(const __grid_constant__ CacheEvictLaunch L) {
  const int h = blockIdx.y, b = blockIdx.z;
  ptx::grid_wait();
  ptx::grid_launch_next();
  fill_page<T, D>(L.out, L.out_k, L.out_v, L.out_mean, b, h, blockIdx.x, KeptTokens(L, b, h), L.status);
}

template <class T, int D>
cudaError_t launch_d(const CacheEvictLaunch& L, cudaStream_t stream) {
  const int problems = L.c.batch * L.c.hkv;
  const int64_t room = static_cast<int64_t>(L.c.max_pages) * L.c.page;
  // What a CTA's registers hold it chooses from alone: both kernels, four heads, 8,192 scores 14.7 us (a cluster of
  // eight 14.4, of two 15.7; eight sequences of them 17.8, with two 20.6), 16,384 31.9 us (eight 15.1). Past what
  // eight hold (65,536 scores) every pass reads them again: a call by itself, its launch and events (7 us) included,
  // 34 us at 65,536, 57 at 65,664, 134 at 262,144.
  const int cluster = choose_cluster(problems, room < L.acc_len ? room : L.acc_len, kChooseThreads * 16, sm_count());
  const cudaError_t e = launch_clusters(cache_evict_choose_kernel, L, problems, kChooseThreads, cluster, stream);
  if (e != cudaSuccess) return e;
  return launch_after(cache_evict_copy_kernel<T, D>, dim3((L.budget + L.out.page - 1) / L.out.page, L.c.hkv, L.c.batch),
                      kPageThreads, 0, stream, L);
}

}  // namespace

cudaError_t launch_cache_evict(const CacheEvictLaunch& L, cudaStream_t stream) {
  if (L.c.dtype == 0) return L.c.head_dim == 128 ? launch_d<BF16, 128>(L, stream) : launch_d<BF16, 64>(L, stream);
  return L.c.head_dim == 128 ? launch_d<FP16, 128>(L, stream) : launch_d<FP16, 64>(L, stream);
}

}  // namespace evisel
