// The highest continuations over a sequence's beams and the vocabulary, in two
// launches: every part of every row of logits gives its maximum, its sum of exponentials
// and its n highest logits; then a CTA per sequence forms the rows' normalisers and
// chooses among the parts' winners.
//
// The n-th largest of the maxima of disjoint groups of elements is a lower bound of
// the n-th largest element: what reaches it is a few more than n elements, which are
// ranked by comparing all with all. Logits are read once; they stay in registers.
#include <algorithm>

#include "cache_common.cuh"
#include "decode_internal.h"

namespace evisel {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kPerThread = 8;                    // 16-byte vectors of a thread
constexpr int kList = 512;                       // elements that reach the bound; beyond, one after the other
constexpr float kLowest = -3.402823466e38f;

struct F32 {};
template <class T>
struct Vec {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& w, float* f) {
    float g[8];
    unpack8<T>(w, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = g[e];
  }
  static __device__ __forceinline__ float one(const void* p, int64_t i) {
    return T::lo(static_cast<const uint16_t*>(p)[i]);
  }
  // A vector of -inf with element e replaced.
  static __device__ __forceinline__ uint32_t minus_inf() { return T::kFormat == 1 ? 0xff80ff80u : 0xfc00fc00u; }
  static __device__ __forceinline__ void load_some(uint4& w, const void* p, int e0, int e1) {
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t none = minus_inf() & 0xffffu;
      const uint32_t lo = 2 * i >= e0 && 2 * i < e1 ? static_cast<const uint16_t*>(p)[2 * i] : none;
      const uint32_t hi = 2 * i + 1 >= e0 && 2 * i + 1 < e1 ? static_cast<const uint16_t*>(p)[2 * i + 1] : none;
      x[i] = lo | hi << 16;
    }
    w = make_uint4(x[0], x[1], x[2], x[3]);
  }
};
template <>
struct Vec<F32> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& w, float* f) {
    f[0] = __uint_as_float(w.x), f[1] = __uint_as_float(w.y), f[2] = __uint_as_float(w.z), f[3] = __uint_as_float(w.w);
  }
  static __device__ __forceinline__ uint32_t minus_inf() { return 0xff800000u; }
  static __device__ __forceinline__ void load_some(uint4& w, const void* p, int e0, int e1) {
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i >= e0 && i < e1 ? static_cast<const uint32_t*>(p)[i] : minus_inf();
    w = make_uint4(x[0], x[1], x[2], x[3]);
  }
};

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}

// Whether (x, i) stands before (y, j): higher, or as high and earlier.
template <class V>
__device__ __forceinline__ bool before(V x, int i, V y, int j) {
  return x > y || (x == y && i < j);
}

// Whether a beam has continuations from its logits.
__device__ __forceinline__ bool beam_is_live(const BeamLaunch& L, int row) {
  if (L.finished && __ldg(L.finished + row)) return false;
  const float s = L.scores ? __ldg(L.scores + row) : 0.f;
  return isfinite(s);
}

// Groups of threads whose maxima bound the n-th largest element.
__device__ __forceinline__ int groups_for(int n) { return n <= 16 ? 64 : n <= 32 ? 128 : 256; }

template <class T>
__global__ void __launch_bounds__(kThreads) beam_scan_kernel(const __grid_constant__ BeamLaunch L) {
  constexpr int N = Vec<T>::N;
  __shared__ __align__(16) float group_max[kThreads];
  __shared__ float list_value[kList], bound;
  __shared__ double warp_total[kWarps];
  __shared__ int list_index[kList], count;
  const int row = blockIdx.y, part = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  ptx::grid_wait();
  ptx::grid_launch_next();
  const int64_t slot = static_cast<int64_t>(row) * L.splits + part;
  if (!beam_is_live(L, row)) return;
  const int b = row / L.beams, k = row - b * L.beams;
  constexpr int kSize = 16 / N;
  const char* base = static_cast<const char*>(L.logits) + (b * L.ls[0] + k * L.ls[1]) * kSize;
  const int skew = static_cast<int>((reinterpret_cast<uintptr_t>(base) & 15) / kSize);   // elements before the row in its first vector
  const uint4* vectors = reinterpret_cast<const uint4*>(base - skew * kSize);
  const int v0 = part * L.part_vectors, v1 = min(v0 + L.part_vectors, (skew + L.vocab + N - 1) / N);
  if (tid == 0) count = 0;

  uint4 w[kPerThread];
  float best = -INFINITY;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    const int v = v0 + tid + i * kThreads;
    w[i] = make_uint4(Vec<T>::minus_inf(), Vec<T>::minus_inf(), Vec<T>::minus_inf(), Vec<T>::minus_inf());
    if (v < v1) {
      const int e0 = skew - v * N, e1 = skew + L.vocab - v * N;   // the row's elements of the vector
      if (e0 <= 0 && e1 >= N) w[i] = __ldg(vectors + v);
      else Vec<T>::load_some(w[i], vectors + v, e0, e1);
    }
  }
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    float x[N];
    Vec<T>::unpack(w[i], x);
#pragma unroll
    for (int e = 0; e < N; ++e) best = fmaxf(best, x[e]);
  }
  const int groups = groups_for(L.n), width = kThreads / groups;
  float g = best;
  for (int o = 1; o < width; o <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, o));
  if (tid % width == 0) group_max[tid / width] = g;
  __syncthreads();

  // The part's maximum, and its sum of exponentials from there.
  float top = -INFINITY;
  for (int i = lane; i < groups; i += 32) top = fmaxf(top, group_max[i]);
  top = warp_max(top);
  const float shift = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    float x[N];
    Vec<T>::unpack(w[i], x);
#pragma unroll
    for (int e = 0; e < N; ++e) sum += ptx::ex2((x[e] - shift) * 1.4426950408889634f);
  }
  double total = sum;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  if (lane == 0) warp_total[warp] = total;
  if (tid < groups) {
    const float mine = group_max[tid];
    int rank = 0;
    for (int i = 0; i < groups; ++i) rank += before(group_max[i], i, mine, tid) ? 1 : 0;
    if (rank == L.n - 1) bound = fmaxf(mine, kLowest);
  }
  __syncthreads();

  if (tid == 0) {
    double s = 0.0;
    for (int i = 0; i < kWarps; ++i) s += warp_total[i];
    L.part_sum[slot] = s;
    L.part_max[slot] = shift;
  }
  const float least = bound;
  if (best >= least) {
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
      float x[N];
      Vec<T>::unpack(w[i], x);
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (x[e] >= least) {
          const int at = atomicAdd(&count, 1);
          if (at < kList) {
            list_value[at] = x[e];
            list_index[at] = (v0 + tid + i * kThreads) * N + e - skew;
          }
        }
    }
  }
  __syncthreads();
  float* value = L.part_value + slot * L.n;
  int32_t* index = L.part_index + slot * L.n;
  const int found = count;
  if (found <= kList) {
    for (int i = tid; i < found; i += kThreads) {
      const float x = list_value[i];
      const int at = list_index[i];
      int rank = 0;
      for (int j = 0; j < found; ++j) rank += before(list_value[j], list_index[j], x, at) ? 1 : 0;
      if (rank < L.n) value[rank] = x, index[rank] = at;
    }
    for (int i = found + tid; i < L.n; i += kThreads) value[i] = -INFINITY, index[i] = -1;
    return;
  }
  // Many as high as one another (a row of few values): the next one after the last, n times.
  float last = INFINITY;
  int last_at = -1;
  for (int r = 0; r < L.n; ++r) {
    float x_best = -INFINITY;
    int at_best = 0x7fffffff;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
      float x[N];
      Vec<T>::unpack(w[i], x);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int at = (v0 + tid + i * kThreads) * N + e - skew;
        if (x[e] > -INFINITY && before(last, last_at, x[e], at) && before(x[e], at, x_best, at_best)) x_best = x[e], at_best = at;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float y = __shfl_xor_sync(0xffffffffu, x_best, o);
      const int yi = __shfl_xor_sync(0xffffffffu, at_best, o);
      if (before(y, yi, x_best, at_best)) x_best = y, at_best = yi;
    }
    __syncthreads();
    if (lane == 0) list_value[warp] = x_best, list_index[warp] = at_best;
    __syncthreads();
    for (int i = 0; i < kWarps; ++i)
      if (before(list_value[i], list_index[i], x_best, at_best)) x_best = list_value[i], at_best = list_index[i];
    last = x_best, last_at = at_best;
    if (tid == 0) value[r] = x_best, index[r] = x_best > -INFINITY ? at_best : -1;
  }
}

// ---------------------------------------------------------------- the choice among the parts' winners
constexpr int kMergeThreads = 512, kMergeWarps = kMergeThreads / 32;
constexpr int kMergeList = 1024;

struct Candidates {
  const BeamLaunch& L;
  const double* offset;             // score - normaliser of a beam; NaN: no continuations from its logits
  int b, per_beam, listed;
  __device__ __forceinline__ int total() const { return listed + L.beams; }
  // Value and flat index (beam, token) of candidate i; -inf where it is none.
  __device__ __forceinline__ void get(int i, double& value, int& flat) const {
    value = -INFINITY;
    flat = 0x7fffffff;
    if (i < listed) {
      const int k = i / per_beam;
      if (!(offset[k] == offset[k])) return;
      const int64_t at = static_cast<int64_t>(b) * listed + i;
      const float x = L.part_value[at];
      if (!(x > -INFINITY)) return;
      value = offset[k] + static_cast<double>(x);
      flat = k * L.vocab + L.part_index[at];
    } else {                                     // an ended beam as it is
      const int k = i - listed, row = b * L.beams + k;
      if (!L.finished || !__ldg(L.finished + row)) return;
      const float s = L.scores ? __ldg(L.scores + row) : 0.f;
      if (!isfinite(s)) return;
      value = s;
      flat = k * L.vocab + L.pad;
    }
  }
};

__global__ void __launch_bounds__(kMergeThreads) beam_merge_kernel(const __grid_constant__ BeamLaunch L) {
  __shared__ double offset[kMaxBeams], group_max[256], list_value[kMergeList], bound;
  __shared__ int list_flat[kMergeList], count;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  ptx::grid_wait();
  ptx::grid_launch_next();
  if (tid == 0) count = 0;
  for (int k = warp; k < L.beams; k += kMergeWarps) {
    const int row = b * L.beams + k;
    const bool live = beam_is_live(L, row);
    double lse = 0.0;
    if (live) {
      const int64_t first = static_cast<int64_t>(row) * L.splits;
      float top = -INFINITY;
      for (int i = lane; i < L.splits; i += 32)
        if (L.part_sum[first + i] != 0.0) top = fmaxf(top, L.part_max[first + i]);
      top = warp_max(top);
      double sum = 0.0;
      for (int i = lane; i < L.splits; i += 32) {
        const double s = L.part_sum[first + i];
        const float m = L.part_max[first + i];
        sum += s == 0.0 ? 0.0 : m == top ? s : s * exp(static_cast<double>(m) - static_cast<double>(top));
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      lse = static_cast<double>(top) + log(sum);
    }
    // A sum that is no number makes every value NaN; a row of -inf has none above it.
    const double score = L.scores ? static_cast<double>(__ldg(L.scores + row)) : 0.0;
    if (lane == 0) offset[k] = live && isfinite(lse) ? score - lse : NAN;
  }
  __syncthreads();
  const Candidates c{L, offset, b, L.splits * L.n, L.beams * L.splits * L.n};
  const int total = c.total(), groups = groups_for(L.n), width = kMergeThreads / groups;
  double best = -INFINITY;
  for (int i = tid; i < total; i += kMergeThreads) {
    double x;
    int f;
    c.get(i, x, f);
    best = fmax(best, x);
  }
  double g = best;
  for (int o = 1; o < width; o <<= 1) g = fmax(g, __shfl_xor_sync(0xffffffffu, g, o));
  if (tid % width == 0) group_max[tid / width] = g;
  __syncthreads();
  if (tid < groups) {
    const double mine = group_max[tid];
    int rank = 0;
    for (int i = 0; i < groups; ++i) rank += before(group_max[i], i, mine, tid) ? 1 : 0;
    if (rank == L.n - 1) bound = fmax(mine, -1.7976931348623157e308);
  }
  __syncthreads();
  const double least = bound;
  if (best >= least)
    for (int i = tid; i < total; i += kMergeThreads) {
      double x;
      int f;
      c.get(i, x, f);
      if (x >= least) {
        const int at = atomicAdd(&count, 1);
        if (at < kMergeList) list_value[at] = x, list_flat[at] = f;
      }
    }
  __syncthreads();
  auto put = [&](int rank, double x, int f) {
    const int64_t at = static_cast<int64_t>(b) * L.n + rank;
    const bool some = x > -INFINITY;
    const int k = some ? f / L.vocab : -1, v = some ? f - k * L.vocab : -1;
    L.score_out[at] = static_cast<float>(x);
    L.parent[at] = k;
    L.token[at] = v;
    if (L.ended_out) L.ended_out[at] = !some || v == L.eos || (L.finished && __ldg(L.finished + b * L.beams + k)) ? 1 : 0;
  };
  const int found = count;
  if (found <= kMergeList) {
    for (int i = tid; i < found; i += kMergeThreads) {
      const double x = list_value[i];
      const int f = list_flat[i];
      int rank = 0;
      for (int j = 0; j < found; ++j) rank += before(list_value[j], list_flat[j], x, f) ? 1 : 0;
      if (rank < L.n) put(rank, x, f);
    }
    for (int i = found + tid; i < L.n; i += kMergeThreads) put(i, -INFINITY, 0);
    return;
  }
  double last = INFINITY;
  int last_flat = -1;
  for (int r = 0; r < L.n; ++r) {
    double x_best = -INFINITY;
    int f_best = 0x7fffffff;
    for (int i = tid; i < total; i += kMergeThreads) {
      double x;
      int f;
      c.get(i, x, f);
      if (x > -INFINITY && before(last, last_flat, x, f) && before(x, f, x_best, f_best)) x_best = x, f_best = f;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const double y = __shfl_xor_sync(0xffffffffu, x_best, o);
      const int yf = __shfl_xor_sync(0xffffffffu, f_best, o);
      if (before(y, yf, x_best, f_best)) x_best = y, f_best = yf;
    }
    __syncthreads();
    if (lane == 0) list_value[warp] = x_best, list_flat[warp] = f_best;
    __syncthreads();
    for (int i = 0; i < kMergeWarps; ++i)
      if (before(list_value[i], list_flat[i], x_best, f_best)) x_best = list_value[i], f_best = list_flat[i];
    last = x_best, last_flat = f_best;
    if (tid == 0) put(r, x_best, f_best);
  }
}

template <class T>
cudaError_t launch_t(const BeamLaunch& L, cudaStream_t stream) {
  const cudaError_t e = launch_after(beam_scan_kernel<T>, dim3(L.splits, L.batch * L.beams), kThreads, 0, stream, L);
  return e != cudaSuccess ? e : launch_after(beam_merge_kernel, dim3(L.batch), kMergeThreads, 0, stream, L);
}

}  // namespace

BeamSplit beam_split(int64_t rows, int vocab, int dtype, int n_sm) {
  const int per = dtype == 2 ? 4 : 8;
  const int vectors = (vocab + per - 1) / per + 1;               // (a row may begin inside one)
  const int most = kThreads * kPerThread;
  int64_t each = (rows * vectors + 2 * n_sm - 1) / (2 * n_sm);   // two CTAs to an SM, where rows are few
  each = std::max<int64_t>(kThreads, std::min<int64_t>(most, (each + kThreads - 1) / kThreads * kThreads));
  BeamSplit s;
  s.splits = static_cast<int>((vectors + each - 1) / each);
  s.part_vectors = (vectors + s.splits - 1) / s.splits;
  return s;
}

cudaError_t launch_beams(const BeamLaunch& L, cudaStream_t stream) {
  return L.dtype == 0 ? launch_t<BF16>(L, stream) : L.dtype == 1 ? launch_t<FP16>(L, stream) : launch_t<F32>(L, stream);
}

}  // namespace evisel
