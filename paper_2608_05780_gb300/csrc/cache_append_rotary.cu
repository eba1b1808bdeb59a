// New tokens into the pages of a cache, their keys rotated on the way, and the
// step's queries: a block per (page that a sequence can touch, head or two), then blocks
// of a warp per token's queries.
//
// A long append is bound by memory as long as enough of it is on its way: 65,664 tokens of four heads (269 MB read and
// written) take 45.6 us, 87% of a plain copy's rate, with 128 threads, five blocks per SM and two heads a block; 52 us with 256
// threads and two blocks, 55 with one head (the angles twice), 77 with the library's sincospif in every head, one
// token of a thread at a time and the means through unpadded columns of shared memory.
// Pages of 16 with eight heads of 64: 57.6 us, 76.8 while half of the threads had no token; one head of 128: 34.6 for half the
// bytes, bound by the angles (formed from a thread's own registers 31.5, but a step's one token of 32 sequences 4.3 for 3.7).
#include "cache_pages.cuh"
#include "rope.cuh"

namespace evisel {
namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32, kBlocks = 5;

// As fill_page(), but D / 16 threads share a token, each with the two pieces of a head that hold its pairs, and a
// block has HEADS heads: two where blocks are many, so that a token's turns are formed once for both, else one and
// two tokens of it at a time. Either way a thread has eight loads on their way. Pages of 16 tokens with heads of 64
// keep half of the threads busy: the other half takes the next heads.
constexpr int groups_of(int d) { return kThreads / (d / 16); }       // of threads, with a token each
template <int D>
__host__ __device__ __forceinline__ int parts_of(int page) { return groups_of(D) > 16 && page == 16 ? 2 : 1; }

template <class T, int D, bool INTER, int HEADS>
__device__ __forceinline__ void fill_page_rotated(const AppendRotaryLaunch& L, int b, int first_head, int page, const NewTokens& src,
                                                  float* mem) {
  constexpr int LANES = D / 16, TOKENS = 2 / HEADS;
  static_assert(groups_of(D) <= 32);             // (two parts at most: pages have 16 tokens or more)
  const CacheView& c = L.a.c;
  const int parts = parts_of<D>(c.page), groups = groups_of(D) / parts, part = threadIdx.x / LANES / groups;
  const int behind = part * HEADS, h0 = first_head + behind;
  const int p0 = page << c.log_page, p1 = min(p0 + c.page, src.end());
  if (p1 <= p0 || p1 <= src.first()) return;     // (the whole block)
  // The page (the heads share a table), which the loads of new tokens need not wait for.
  const int64_t id = __ldg(c.table + b * c.ts[0] + page);
  uint16_t* k = static_cast<uint16_t*>(const_cast<void*>(c.k)) + h0 * c.ks[1];
  uint16_t* v = static_cast<uint16_t*>(const_cast<void*>(c.v)) + h0 * c.vs[1];
  const int j = threadIdx.x % LANES, grp = threadIdx.x / LANES - part * groups;
  const bool rotates = 8 * j < L.rope.pairs;
  int lo, hi;
  lane_pieces(L.rope, j, lo, hi);
  float sum_lo[HEADS][8] = {}, sum_hi[HEADS][8] = {};
  for (int base = h0 < c.hkv ? p0 + grp : p1; base < p1; base += groups * TOKENS) {
    uint4 a[2], w[2], x[2], y[2];
    bool fresh[TOKENS], in[TOKENS];
    int at[TOKENS][3];
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
      const int pos = base + t * groups;
      fresh[t] = pos < p1 && pos >= src.first();
      in[t] = fresh[t] || (pos < p1 && c.k_mean);                  // an older token is read for the mean only
      const int i = fresh[t] ? src.token(pos) : 0;
#pragma unroll
      for (int u = 0; u < HEADS; ++u) {
        const int n = t * HEADS + u;
        a[n] = w[n] = make_uint4(0, 0, 0, 0);
        if (fresh[t]) {
          const uint4 *kr = src.key(i, behind + u), *vr = src.value(i, behind + u);
          a[n] = kr[lo], w[n] = kr[hi], x[n] = vr[lo], y[n] = vr[hi];
        }
      }
      if (fresh[t] && rotates) positions_of(L.rope, L.pos, b, i, src.len, pos - src.len, at[t]);
    }
    if (static_cast<uint64_t>(id) >= static_cast<uint64_t>(c.n_pages)) break;
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
      const int slot = base + t * groups - p0;
      if (in[t] && !fresh[t]) {
#pragma unroll
        for (int u = 0; u < HEADS; ++u) {
          const uint4* kr = reinterpret_cast<const uint4*>(k + id * c.ks[0] + u * c.ks[1] + slot * c.ks[2]);
          a[t * HEADS + u] = kr[lo], w[t * HEADS + u] = kr[hi];
        }
      }
      if (fresh[t]) {
        if (rotates) {
          float2 cs[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) cs[e] = pair_turn(L.rope, at[t], 8 * j + e, 1.f);
#pragma unroll
          for (int u = 0; u < HEADS; ++u) rotate_pieces<T, INTER>(a[t * HEADS + u], w[t * HEADS + u], cs);
        }
#pragma unroll
        for (int u = 0; u < HEADS; ++u) {
          const int n = t * HEADS + u;
          uint4* kd = reinterpret_cast<uint4*>(k + id * c.ks[0] + u * c.ks[1] + slot * c.ks[2]);
          uint4* vd = reinterpret_cast<uint4*>(v + id * c.vs[0] + u * c.vs[1] + slot * c.vs[2]);
          kd[lo] = a[n], kd[hi] = w[n], vd[lo] = x[n], vd[hi] = y[n];
        }
      }
#pragma unroll
      for (int u = 0; u < HEADS; ++u) {
        float f[8], g[8];
        unpack8<T>(a[t * HEADS + u], f);
        unpack8<T>(w[t * HEADS + u], g);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum_lo[u][e] += f[e], sum_hi[u][e] += g[e];
      }
    }
  }
  if (static_cast<uint64_t>(id) >= static_cast<uint64_t>(c.n_pages)) {             // (every thread: some have no token)
    record_bounds(L.a.status);
    return;
  }
  if (!c.k_mean) return;
  // A warp's tokens by shuffles, the warps' sums through shared memory.
  const int warps = kWarps / parts;              // of a part
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int u = 0; u < HEADS; ++u) {
#pragma unroll
    for (int o = LANES; o < 32; o <<= 1)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sum_lo[u][e] += __shfl_xor_sync(0xffffffffu, sum_lo[u][e], o);
        sum_hi[u][e] += __shfl_xor_sync(0xffffffffu, sum_hi[u][e], o);
      }
    if (lane < LANES) {
      float4* m = reinterpret_cast<float4*>(mem + ((behind + u) * warps + warp - part * warps) * D);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        m[lo * 2 + e] = make_float4(sum_lo[u][4 * e], sum_lo[u][4 * e + 1], sum_lo[u][4 * e + 2], sum_lo[u][4 * e + 3]);
        m[hi * 2 + e] = make_float4(sum_hi[u][4 * e], sum_hi[u][4 * e + 1], sum_hi[u][4 * e + 2], sum_hi[u][4 * e + 3]);
      }
    }
  }
  __syncthreads();
  const float n = static_cast<float>(p1 - p0);
  uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(const_cast<void*>(c.k_mean)) + (id * c.hkv + first_head) * D);
  for (int i = threadIdx.x; i < min(HEADS * parts, c.hkv - first_head) * (D / 2); i += kThreads) {
    const float* m = mem + (i / (D / 2) * warps) * D + i % (D / 2) * 2;
    float p = 0.f, q = 0.f;
#pragma unroll
    for (int g = 0; g < kWarps; ++g)
      if (g < warps) p += m[g * D], q += m[g * D + 1];
    dst[i] = T::pack(p / n, q / n);
  }
}

template <class T, int D, bool INTER, int HEADS>
__global__ void __launch_bounds__(kThreads, kBlocks) cache_append_rotary_kernel(const __grid_constant__ AppendRotaryLaunch L, int pages,
                                                                           int share, int shares) {
  __shared__ __align__(16) float mem[kThreads * 16];
  const CacheView& c = L.a.c;
  const int heads = HEADS * parts_of<D>(c.page), head_blocks = (c.hkv + heads - 1) / heads;
  const int64_t kv_blocks = static_cast<int64_t>(pages) * head_blocks * c.batch;
  ptx::grid_wait();
  ptx::grid_launch_next();
  if (blockIdx.x < kv_blocks) {
    const int x = blockIdx.x % pages, bh = blockIdx.x / pages, b = bh / head_blocks, h = (bh - b * head_blocks) * heads;
    const NewTokens src(L.a, b, h);
    if (x == 0 && h == 0 && threadIdx.x == 0) L.a.lens_out[b] = src.end();
    fill_page_rotated<T, D, INTER, HEADS>(L, b, h, (src.len >> c.log_page) + x, src, mem);
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
  const int heads = L.a.c.hkv % 2 == 0 && grid >= kBlocks * 2 * static_cast<int64_t>(sm_count()) ? 2 : 1;
  const int block_heads = heads * parts_of<D>(L.a.c.page);
  grid = static_cast<int64_t>(pages) * ((L.a.c.hkv + block_heads - 1) / block_heads) * L.a.c.batch;
  int share = 1, shares = 1;
  if (L.q.heads > 0 && rows > 0) {
    share = rotary_heads_per_warp(rows, L.q.heads, D, sm_count());
    shares = (L.q.heads + share - 1) / share;
    grid += (rows * shares + kWarps - 1) / kWarps;
  }
  if (grid > 0x7fffffff) return cudaErrorInvalidConfiguration;
  const auto kernel = heads == 2 ? (L.rope.interleaved ? cache_append_rotary_kernel<T, D, true, 2> : cache_append_rotary_kernel<T, D, false, 2>)
                                 : (L.rope.interleaved ? cache_append_rotary_kernel<T, D, true, 1> : cache_append_rotary_kernel<T, D, false, 1>);
  return launch_after(kernel, dim3(static_cast<unsigned>(grid)), kThreads, 0, stream, L, pages, share, shares);
}

}  // namespace

cudaError_t launch_append_rotary(const AppendRotaryLaunch& L, cudaStream_t stream) {
  if (L.a.c.dtype == 0) return L.a.c.head_dim == 128 ? launch_d<BF16, 128>(L, stream) : launch_d<BF16, 64>(L, stream);
  return L.a.c.head_dim == 128 ? launch_d<FP16, 128>(L, stream) : launch_d<FP16, 64>(L, stream);
}

}  // namespace evisel
