// New tokens into the pages of a cache, their keys rotated on the way, and the
// step's queries: a block per (page that a sequence can touch, head), then blocks
// of a warp per token's queries.
#include "cache_pages.cuh"
#include "rope.cuh"

namespace evisel {
namespace {

constexpr int kWarps = kPageThreads / 32;

// As fill_page(), but D / 16 threads share a token, each with the two pieces of a
// head that hold its pairs.
template <class T, int D, bool INTER>
__device__ __forceinline__ void fill_page_rotated(const AppendRotaryLaunch& L, int b, int h, int page, const NewTokens& src,
                                                  float* mem) {
  constexpr int LANES = D / 16, GROUPS = kPageThreads / LANES;
  const CacheView& c = L.a.c;
  const int p0 = page << c.log_page, p1 = min(p0 + c.page, src.end());
  if (p1 <= p0 || p1 <= src.first()) return;     // (the whole block)
  const int64_t id = cache_page_to_write(c, b, h, page, L.a.status);
  if (id < 0) return;
  uint16_t* k = static_cast<uint16_t*>(const_cast<void*>(c.k)) + id * c.ks[0] + h * c.ks[1];
  uint16_t* v = static_cast<uint16_t*>(const_cast<void*>(c.v)) + id * c.vs[0] + h * c.vs[1];
  const int j = threadIdx.x % LANES, grp = threadIdx.x / LANES;
  int lo, hi;
  lane_pieces(L.rope, j, lo, hi);
  float sum_lo[8] = {}, sum_hi[8] = {};
  for (int slot = grp; p0 + slot < p1; slot += GROUPS) {
    const int pos = p0 + slot;
    uint4* kd = reinterpret_cast<uint4*>(k + slot * c.ks[2]);
    uint4 a, w;
    if (pos >= src.first()) {
      const int i = src.token(pos);
      const uint4 *kr = src.key(i), *vr = src.value(i);
      a = kr[lo], w = kr[hi];
      const uint4 x = vr[lo], y = vr[hi];
      if (8 * j < L.rope.pairs) {
        int at[3];
        positions_of(L.rope, L.pos, b, i, src.len, pos - src.len, at);
        float2 cs[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) cs[e] = pair_turn(L.rope, at, 8 * j + e, 1.f);
        rotate_pieces<T, INTER>(a, w, cs);
      }
      uint4* vd = reinterpret_cast<uint4*>(v + slot * c.vs[2]);
      kd[lo] = a, kd[hi] = w, vd[lo] = x, vd[hi] = y;
    } else if (c.k_mean) {
      a = kd[lo], w = kd[hi];                    // an older token, for the mean
    } else {
      continue;
    }
    float f[8], g[8];
    unpack8<T>(a, f);
    unpack8<T>(w, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum_lo[e] += f[e], sum_hi[e] += g[e];
  }
  if (!c.k_mean) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) mem[grp * D + lo * 8 + e] = sum_lo[e], mem[grp * D + hi * 8 + e] = sum_hi[e];
  __syncthreads();
  const float n = static_cast<float>(p1 - p0);
  uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(const_cast<void*>(c.k_mean)) + (id * c.hkv + h) * D);
  for (int i = threadIdx.x; i < D / 2; i += kPageThreads) {
    float x = 0.f, y = 0.f;
    for (int g = 0; g < GROUPS; ++g) x += mem[g * D + 2 * i], y += mem[g * D + 2 * i + 1];
    dst[i] = T::pack(x / n, y / n);
  }
}

template <class T, int D, bool INTER>
__global__ void __launch_bounds__(kPageThreads) cache_append_rotary_kernel(const __grid_constant__ AppendRotaryLaunch L, int pages,
                                                                           int share, int shares) {
  __shared__ __align__(16) float mem[kPageThreads * 16];
  const CacheView& c = L.a.c;
  const int64_t kv_blocks = static_cast<int64_t>(pages) * c.hkv * c.batch;
  ptx::grid_wait();
  ptx::grid_launch_next();
  if (blockIdx.x < kv_blocks) {
    const int x = blockIdx.x % pages, bh = blockIdx.x / pages, b = bh / c.hkv, h = bh - b * c.hkv;
    const NewTokens src(L.a, b, h);
    if (x == 0 && h == 0 && threadIdx.x == 0) L.a.lens_out[b] = src.end();
    fill_page_rotated<T, D, INTER>(L, b, h, (src.len >> c.log_page) + x, src, mem);
    return;
  }
  const int warp = threadIdx.x >> 5;
  const int64_t item = (static_cast<int64_t>(blockIdx.x) - kv_blocks) * kWarps + warp, n = item / shares;
  if (n >= static_cast<int64_t>(c.batch) * L.a.d.tokens) return;
  const int b = static_cast<int>(n / L.a.d.tokens), t = static_cast<int>(n - static_cast<int64_t>(b) * L.a.d.tokens);
  const int h0 = static_cast<int>(item - n * shares) * share;
  int pos[3];
  positions_of(L.rope, L.pos, b, t, L.pos.at || L.pos.first ? 0 : cache_len(c, b, 0, L.a.status), t, pos);
  rotate_token<T, D, INTER>(L.rope, L.q, HeadsView{}, b, t, pos, 1.f, h0, min(L.q.heads, h0 + share),
                            reinterpret_cast<float2*>(mem) + warp * (D / 2));
}

template <class T, int D>
cudaError_t launch_d(const AppendRotaryLaunch& L, cudaStream_t stream) {
  const int tokens = L.a.d.tokens;
  const int pages = (tokens + L.a.c.page - 1) / L.a.c.page + 1;  // that T tokens can touch
  const int64_t rows = static_cast<int64_t>(L.a.c.batch) * tokens;
  int64_t grid = static_cast<int64_t>(pages) * L.a.c.hkv * L.a.c.batch;
  int share = 1, shares = 1;
  if (L.q.heads > 0 && rows > 0) {
    share = rotary_heads_per_warp(rows, L.q.heads, D, sm_count());
    shares = (L.q.heads + share - 1) / share;
    grid += (rows * shares + kWarps - 1) / kWarps;
  }
  if (grid > 0x7fffffff) return cudaErrorInvalidConfiguration;
  return launch_after(L.rope.interleaved ? cache_append_rotary_kernel<T, D, true> : cache_append_rotary_kernel<T, D, false>,
                      dim3(static_cast<unsigned>(grid)), kPageThreads, 0, stream, L, pages, share, shares);
}

}  // namespace

cudaError_t launch_append_rotary(const AppendRotaryLaunch& L, cudaStream_t stream) {
  if (L.a.c.dtype == 0) return L.a.c.head_dim == 128 ? launch_d<BF16, 128>(L, stream) : launch_d<BF16, 64>(L, stream);
  return L.a.c.head_dim == 128 ? launch_d<FP16, 128>(L, stream) : launch_d<FP16, 64>(L, stream);
}

}  // namespace evisel
