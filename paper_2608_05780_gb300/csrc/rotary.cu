// Position rotation of queries and keys: every element read and written once, a warp
// to a token (or, where tokens are few, to some of its heads), whose lanes form the token's turns once.
// The stream is the bound: 65,664 tokens of 28 + 4 heads of 128 (1.08 GB read and written) in 154 us, as fast as a
// plain copy; a few tokens take 2.7 us, a launch and dependent loads. A token's heads are read before its turns are formed (40,000
// tokens of 16 + 8 heads of 64: 39.8 us, 43.6 after them). Few heads are latency: 4 + 2 of 64, 20 us of which 9 are the stream,
// 26.6 with the registers for four times as many; several tokens to a warp were 23, their places cost more than they hide.
#include "rope.cuh"

namespace evisel {
namespace {

constexpr int kWarps = 8;

template <class T, int D, bool INTER, int AT>
__global__ void __launch_bounds__(kWarps * 32, AT == 4 ? 3 : AT == 2 ? 4 : 5) rotary_kernel(const __grid_constant__ RotaryLaunch L, int share, int shares) {
  __shared__ float2 mem[kWarps][D / 2];
  const int warp = threadIdx.x >> 5;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * kWarps + warp;
  ptx::grid_wait();
  ptx::grid_launch_next();
  const int64_t n = item / shares;
  if (n >= static_cast<int64_t>(L.batch) * L.tokens) return;
  const int b = static_cast<int>(n / L.tokens), t = static_cast<int>(n - static_cast<int64_t>(b) * L.tokens);
  const int heads = L.q.heads + L.k.heads, h0 = static_cast<int>(item - n * shares) * share;
  int pos[3];
  positions_of(L.rope, L.pos, b, t, 0, t, pos);
  rotate_token<T, D, INTER, AT>(L.rope, L.q, L.k, b, t, pos, L.transpose ? -1.f : 1.f, h0, min(heads, h0 + share), mem[warp]);
}

template <class T, int D>
cudaError_t launch_d(const RotaryLaunch& L, cudaStream_t stream) {
  const int64_t tokens = static_cast<int64_t>(L.batch) * L.tokens;
  const int heads = L.q.heads + L.k.heads, share = rotary_heads_per_warp(tokens, heads, D, sm_count());
  const int shares = (heads + share - 1) / share;
  const unsigned grid = static_cast<unsigned>((tokens * shares + kWarps - 1) / kWarps);
  // As many heads at a time as a warp has passes (6 + 2 heads of 128 at 40,000 tokens: 31.5 us with two passes at a time, 36 with four).
  const int passes = share * D / 512;
  const auto kernel = L.rope.interleaved ? (passes <= 1 ? rotary_kernel<T, D, true, 1> : passes <= 2 ? rotary_kernel<T, D, true, 2> : rotary_kernel<T, D, true, 4>)
                                         : (passes <= 1 ? rotary_kernel<T, D, false, 1> : passes <= 2 ? rotary_kernel<T, D, false, 2> : rotary_kernel<T, D, false, 4>);
  return launch_after(kernel, dim3(grid), kWarps * 32, 0, stream, L, share, shares);
}

}  // namespace

cudaError_t launch_rotary(const RotaryLaunch& L, cudaStream_t stream) {
  if (L.dtype == 0) return L.head_dim == 128 ? launch_d<BF16, 128>(L, stream) : launch_d<BF16, 64>(L, stream);
  return L.head_dim == 128 ? launch_d<FP16, 128>(L, stream) : launch_d<FP16, 64>(L, stream);
}

}  // namespace evisel
