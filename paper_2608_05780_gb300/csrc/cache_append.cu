// New tokens into the pages of a cache, a block per page that they can touch.
// The stream is the bound: 65,664 tokens (269 MB, read and written) in 41 us, 97% of a plain copy's rate.
#include <cstdint>
#include <cuda_runtime.h>

#include "cache_pages.cuh"

namespace evisel {
namespace {

struct NewTokens {
  const CacheAppendLaunch& L;
  int b, h, len, count;
  __device__ __forceinline__ NewTokens(const CacheAppendLaunch& L_, int b_, int h_) : L(L_), b(b_), h(h_) {
    len = cache_len(L.c, b, 0, L.status);
    count = L.counts ? __ldg(L.counts + b) : L.d.tokens;
    const int64_t room = (static_cast<int64_t>(L.c.max_pages) << L.c.log_page) - len;
    if (count < 0 || count > L.d.tokens || count > room) {
      record_bounds(L.status);
      count = count < 0 ? 0 : static_cast<int>(min(static_cast<int64_t>(min(count, L.d.tokens)), room));
    }
    if (__ldg(L.c.lens + b * L.c.ls[0]) < 0) count = 0;   // the first pages may be another sequence's too
  }
  __device__ __forceinline__ int first() const { return len; }
  __device__ __forceinline__ int end() const { return len + count; }
  __device__ __forceinline__ void rows(int pos, const uint4*& k, const uint4*& v) const {
    int i = pos - len;
    if (L.src) {
      i = __ldg(L.src + static_cast<int64_t>(b) * L.d.tokens + i);
      if (static_cast<unsigned>(i) >= static_cast<unsigned>(L.d.tokens)) {
        record_bounds(L.status);
        i = 0;
      }
    }
    k = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(L.d.k_new) + b * L.d.kns[0] + i * L.d.kns[1] + h * L.d.kns[2]);
    v = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(L.d.v_new) + b * L.d.vns[0] + i * L.d.vns[1] + h * L.d.vns[2]);
  }
};

template <class T, int D>
__global__ void __launch_bounds__(kPageThreads, kPageBlocks) cache_append_kernel(const __grid_constant__ CacheAppendLaunch L) {
  const int h = blockIdx.y, b = blockIdx.z;
  ptx::grid_wait();
  ptx::grid_launch_next();
  const NewTokens src(L, b, h);
  if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) L.lens_out[b] = src.end();
  fill_page<T, D>(L.c, const_cast<void*>(L.c.k), const_cast<void*>(L.c.v), const_cast<void*>(L.c.k_mean), b, h,
                  (src.len >> L.c.log_page) + blockIdx.x, src, L.status);
}

template <class T, int D>
cudaError_t launch_d(const CacheAppendLaunch& L, cudaStream_t stream) {
  const int pages = (L.d.tokens + L.c.page - 1) / L.c.page + 1;  // that T tokens can touch
  return launch_after(cache_append_kernel<T, D>, dim3(pages, L.c.hkv, L.c.batch), kPageThreads, 0, stream, L);
}

}  // namespace

cudaError_t launch_cache_append(const CacheAppendLaunch& L, cudaStream_t stream) {
  if (L.c.dtype == 0) return L.c.head_dim == 128 ? launch_d<BF16, 128>(L, stream) : launch_d<BF16, 64>(L, stream);
  return L.c.head_dim == 128 ? launch_d<FP16, 128>(L, stream) : launch_d<FP16, 64>(L, stream);
}

}  // namespace evisel
