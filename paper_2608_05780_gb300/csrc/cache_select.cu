// Pages chosen for the queries of a (sequence, KV head) by their mean keys:
//   score_j = max over the rows of q . k_mean_j.
//
// One launch, a cluster of CTAs per (sequence, KV head): each CTA forms the scores
// of its part of the pages (16 pages against 8 rows per mma.sync, both read from
// global memory 16 bytes a lane, the products' order along d permuted alike on
// both sides) in shared memory, takes the others' over, chooses among all of them
// and writes what falls into its part: one exchange, where a choice over the
// cluster's histograms takes one per digit. Latency is the bound: 64 of up to 1,026
// pages of eight sequences, one token of 7 heads, 9 us for 8 MB of means.
#include <cstdint>
#include <cuda_runtime.h>

#include "cache_choose.cuh"

namespace evisel {
namespace {

constexpr int kChooseThreads = 512;
constexpr int kMaxPages = 8192;                  // scores of a (sequence, KV head), over its cluster
constexpr float kNone = -INFINITY;

template <class T, int D>
__global__ void __launch_bounds__(kChooseThreads) cache_select_kernel(const __grid_constant__ CacheSelectLaunch L) {
  __shared__ ChooseMem mem;
  __shared__ uint32_t score[kMaxPages];          // order keys of the pages from lo on
  ptx::grid_wait();
  ptx::grid_launch_next();
  constexpr int J = D / 32;                      // 16-byte chunks of a row per lane
  const int rank = static_cast<int>(ptx::cluster_rank()), size = static_cast<int>(ptx::cluster_size());
  const int problem = blockIdx.x / size, b = problem / L.c.hkv, h = problem % L.c.hkv;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, fr = lane >> 2, fc = (lane & 3) * 8;
  const int len = cache_len(L.c, b, h, L.status), n = (len + L.c.page - 1) >> L.c.log_page;
  const int count = min(n, L.n_select);
  const bool all = n <= L.n_select;
  const int sink = all ? count : L.sink, recent = all ? 0 : L.recent, want = count - sink - recent;
  const int lo = sink, hi = n - recent;
  const ChoosePart part(lo, hi, rank, size);

  if (want > 0) {
    const int rows = drafted_tokens(L.d, b) * L.d.gq, n_part = part.b - part.a;
    for (int i = threadIdx.x; i < n_part; i += kChooseThreads) score[part.a - lo + i] = order_key(-INFINITY);
    __syncthreads();
    // Tasks of 16 pages against a share of the rows, so many shares that every warp has a task.
    const int page_tiles = (n_part + 15) / 16, row_tiles = (rows + 7) / 8;
    const int shares = page_tiles > 0 ? min(row_tiles, (kChooseThreads / 32 + page_tiles - 1) / page_tiles) : 0;
    const uint16_t* q0 = static_cast<const uint16_t*>(L.d.q) + b * L.d.qs[0] + h * L.d.gq * L.d.qs[2] + fc;
    for (int task = warp; task < page_tiles * shares; task += kChooseThreads / 32) {
      const int p0 = part.a + task / shares * 16, share = task % shares;
      const int first_row = row_tiles * share / shares * 8, end_row = min(rows, row_tiles * (share + 1) / shares * 8);
      uint4 a[2][J];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int p = min(p0 + fr + 8 * half, part.b - 1);       // past the part: its last page again, not kept
        const int64_t id = cache_page(L.c, b, h, p, L.status);
        const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(L.c.k_mean) + (id * L.c.hkv + h) * D + fc);
#pragma unroll
        for (int j = 0; j < J; ++j) a[half][j] = __ldg(src + 4 * j);
      }
      float top[2] = {kNone, kNone};
#pragma unroll 2
      for (int r0 = first_row; r0 < end_row; r0 += 8) {
        const int r = min(r0 + fr, rows - 1), t = r / L.d.gq, g = r % L.d.gq;   // past the rows: the last one again
        const uint4* src = reinterpret_cast<const uint4*>(q0 + t * L.d.qs[1] + g * L.d.qs[2]);
        float c[4] = {};
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const uint4 x = __ldg(src + 4 * j);
          const uint32_t f0[4] = {a[0][j].x, a[1][j].x, a[0][j].y, a[1][j].y};
          const uint32_t f1[4] = {a[0][j].z, a[1][j].z, a[0][j].w, a[1][j].w};
          ptx::mma16816<T>(c, f0, x.x, x.y);
          ptx::mma16816<T>(c, f1, x.z, x.w);
        }
        top[0] = fmaxf(top[0], fmaxf(c[0], c[1]));
        top[1] = fmaxf(top[1], fmaxf(c[2], c[3]));
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        top[half] = fmaxf(top[half], __shfl_xor_sync(0xffffffffu, top[half], 1));
        top[half] = fmaxf(top[half], __shfl_xor_sync(0xffffffffu, top[half], 2));
        const int p = p0 + fr + 8 * half;
        // (the order of the maxima does not matter: the keys are whole numbers)
        if ((lane & 3) == 0 && p < part.b) atomicMax(&score[p - lo], order_key(top[half]));
      }
    }
    if (size > 1) {
      ptx::cluster_sync();
      for (int i = threadIdx.x; i < hi - lo; i += kChooseThreads) {
        const int owner = i / max(1, part.chunk);
        if (owner != rank) score[i] = static_cast<uint32_t>(ptx::ld_cluster(ptx::smem_addr(&score[i]), owner));
      }
    }
    __syncthreads();
  }

  const int64_t at = static_cast<int64_t>(problem) * L.n_select;
  auto put = [&](int place, int page) {
    L.pages[at + place] = page;
    L.sel_table[at + place] = cache_page(L.c, b, h, page, L.status);
  };
  const int first = rank * kChooseThreads + static_cast<int>(threadIdx.x), step = size * kChooseThreads;
  for (int i = first; i < sink; i += step) put(i, i);
  for (int i = first; i < recent; i += step) put(count - recent + i, n - recent + i);
  for (int i = count + first; i < L.n_select; i += step) L.pages[at + i] = L.sel_table[at + i] = -1;
  choose_top<kChooseThreads, 4>(lo, hi, want, [&](int i) { return score[i - lo]; }, mem,
                                [&](int place, int i) {
                                  if (i >= part.a && i < part.b) put(sink + place, i);
                                }, 0, 1, [] {});
  if (first == 0) L.sel_lens[problem] = count > 0 ? (count - 1) * L.c.page + (len - (n - 1) * L.c.page) : 0;
  if (size > 1) ptx::cluster_sync();
}

template <class T, int D>
cudaError_t launch_d(const CacheSelectLaunch& L, cudaStream_t stream) {
  // By the products of 8 rows with a page's mean: 256 (256 pages, one token of 7 heads) take 5.8 us alone and 6.1 in
  // clusters of eight, 512 7.7 and 6.7, 896 (128 pages, eight tokens) 7.5 and 6.9, 57,344 110 and 21.
  const int problems = L.c.batch * L.c.hkv, row_tiles = (L.d.tokens * L.d.gq + 7) / 8;
  const int cluster = choose_cluster(problems, static_cast<int64_t>(L.c.max_pages) * row_tiles, 384, sm_count());
  return launch_clusters(cache_select_kernel<T, D>, L, problems, kChooseThreads, cluster, stream);
}

}  // namespace

cudaError_t launch_cache_select(const CacheSelectLaunch& L, cudaStream_t stream) {
  if (L.c.dtype == 0) return L.c.head_dim == 128 ? launch_d<BF16, 128>(L, stream) : launch_d<BF16, 64>(L, stream);
  return L.c.head_dim == 128 ? launch_d<FP16, 128>(L, stream) : launch_d<FP16, 64>(L, stream);
}

}  // namespace evisel
