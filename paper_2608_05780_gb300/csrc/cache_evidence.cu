// Attention weight per cached token:
//   acc[b, h, m] (+)= sum_{t used} sum_{heads g of group h} exp(scale q . k_m - LSE).
// One thread per key: its key in registers, the rows' queries by broadcast loads.
#include <cstdint>
#include <cuda_runtime.h>

#include "cache_common.cuh"

namespace evisel {
namespace {

constexpr int kThreads = 128;
constexpr float kLog2e = 1.4426950408889634f;

template <class T, int D>
__global__ void __launch_bounds__(kThreads) cache_evidence_kernel(const __grid_constant__ CacheEvidenceLaunch L) {
  const int h = blockIdx.y, b = blockIdx.z, key = blockIdx.x * kThreads + threadIdx.x;
  int len = cache_len(L.c, b, h, L.status);
  if (len > L.acc_len) {
    record_bounds(L.status);
    len = static_cast<int>(L.acc_len);
  }
  if (key >= len) return;
  const int id = cache_page(L.c, b, h, key >> L.c.log_page, L.status);
  const uint4* k = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(L.c.k) + id * L.c.ks[0] + h * L.c.ks[1] +
                                                  (key & (L.c.page - 1)) * L.c.ks[2]);
  uint4 kr[D / 8];
#pragma unroll
  for (int i = 0; i < D / 8; ++i) kr[i] = __ldg(k + i);
  const int drafted = drafted_tokens(L.d, b);
  float sum = 0.f;
  for (int t = 0; t < drafted; ++t) {
    if (L.use && !__ldg(L.use + static_cast<int64_t>(b) * L.d.tokens + t)) continue;
    for (int g = 0; g < L.d.gq; ++g) {
      const int head = h * L.d.gq + g;
      const float lse = __ldg(L.lse + (static_cast<int64_t>(head) * L.c.batch + b) * L.d.tokens + t);
      if (lse == -INFINITY) continue;
      const uint4* q = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(L.d.q) + b * L.d.qs[0] +
                                                      t * L.d.qs[1] + head * L.d.qs[2]);
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        float x[8], y[8];
        unpack8<T>(kr[i], x);
        unpack8<T>(__ldg(q + i), y);
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(x[e], y[e], s);
      }
      sum += ptx::ex2(fmaf(s, L.d.scale_log2, -kLog2e * lse));
    }
  }
  float* dst = L.acc + (static_cast<int64_t>(b) * L.c.hkv + h) * L.acc_len + key;
  *dst = L.accumulate ? *dst + sum : sum;
}

template <class T, int D>
cudaError_t launch_d(const CacheEvidenceLaunch& L, cudaStream_t stream) {
  const int64_t room = static_cast<int64_t>(L.c.max_pages) * L.c.page;
  const dim3 grid(static_cast<unsigned>((room + kThreads - 1) / kThreads), L.c.hkv, L.c.batch);
  cache_evidence_kernel<T, D><<<grid, kThreads, 0, stream>>>(L);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_cache_evidence(const CacheEvidenceLaunch& L, cudaStream_t stream) {
  if (L.c.dtype == 0) return L.c.head_dim == 128 ? launch_d<BF16, 128>(L, stream) : launch_d<BF16, 64>(L, stream);
  return L.c.head_dim == 128 ? launch_d<FP16, 128>(L, stream) : launch_d<FP16, 64>(L, stream);
}

}  // namespace evisel
