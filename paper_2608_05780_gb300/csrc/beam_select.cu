// The highest continuations over a sequence's beams and the vocabulary, in two
// launches (or, of few logits, one). A row of logits is cut into blocks of 1,024 tokens (512 in 32 bits; powers of two more for
// long rows); a warp streams a block and leaves its maximum and its sum of exponentials. Then a CTA per sequence forms
// the rows' normalisers from the blocks' sums, takes the n highest blocks by where their highest continuations
// stand (their values, then beam, logit and place: different logits may have the same value), in which
// all of the n highest continuations lie, and reads those again: for any
// continuation outside, each of the n blocks has one that stands before it.
//
// So the pass over the logits keeps no lists, and warps wait for nothing but their loads. What it costs beside the
// memory is instructions: 64 sequences of 8 beams over 152,064 tokens (156 MB) take 25.5 us (6.1 TB/s, 90% of a plain copy's rate,
// the schedulers 71% busy), 29.5 with two divisions a block, 42 with lists of candidates by CTA and their bounds.
// The choice is a chain of dependent steps: 6.5 us more there, 4.5 of the 6.5 us that four beams over 32,000 tokens take.
#include <algorithm>

#include "cache_choose.cuh"
#include "cache_common.cuh"
#include "decode_internal.h"

namespace evisel {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32, kPerSm = 2;
constexpr int kCluster = 8, kSmallBlocks = 2;     // CTAs of a sequence whose blocks are few: so many to a warp at most
constexpr int kPerLane = 4;                      // 16-byte vectors of a lane's chunk; the next chunk is in flight
constexpr int kChunkShift = 7, kChunk = 32 * kPerLane;
static_assert(kChunk == 1 << kChunkShift);
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLog2eLow = 1.925963033500e-8f;  // log2 e - kLog2e

__device__ __forceinline__ uint4 load_once(const uint4* p) {
  uint4 w;
  asm volatile("ld.global.nc.L1::no_allocate.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "l"(p));
  return w;
}

// The 16 bytes that begin `by` words (0 to 3) into a and end in b.
__device__ __forceinline__ uint4 shifted_words(uint4 a, uint4 b, int by) {
  if (by & 2) a = make_uint4(a.z, a.w, b.x, b.y), b = make_uint4(b.z, b.w, 0, 0);
  if (by & 1) a = make_uint4(a.y, a.z, a.w, b.x);
  return a;
}

struct F32 {};
template <class T>
struct Vec {
  static constexpr int N = 8;
  static constexpr uint32_t kNone = T::kFormat == 1 ? 0xff80ff80u : 0xfc00fc00u;   // -inf twice
  static __device__ __forceinline__ void unpack(const uint4& w, float (&f)[8]) { unpack8<T>(w, f); }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    if constexpr (T::kFormat == 1)
      asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else
      asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ float element(const uint4* p, int i) { return T::lo(__ldg(reinterpret_cast<const uint16_t*>(p) + i)); }
  static __device__ __forceinline__ float highest(const uint4& w) {
    const uint32_t m = max2(max2(w.x, w.y), max2(w.z, w.w));
    return fmaxf(T::lo(m), T::hi(m));
  }
  // The largest of the vectors' elements.
  static __device__ __forceinline__ float highest(const uint4 (&w)[kPerLane]) {
    uint32_t m = kNone;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) m = max2(m, max2(max2(w[i].x, w[i].y), max2(w[i].z, w[i].w)));
    return fmaxf(T::lo(m), T::hi(m));
  }
  // The vector that begins `by` elements into a (by < N) and ends in b.
  static __device__ __forceinline__ uint4 shifted(const uint4& a, const uint4& b, int by) {
    const uint4 w = shifted_words(a, b, by >> 1);
    const uint32_t x = shifted_words(b, b, by >> 1).x;             // the word behind
    const uint32_t bits = (by & 1) * 16;
    return make_uint4(__funnelshift_r(w.x, w.y, bits), __funnelshift_r(w.y, w.z, bits), __funnelshift_r(w.z, w.w, bits),
                      __funnelshift_r(w.w, x, bits));
  }
  // The elements [e0, e1) of a vector, -inf beside them.
  static __device__ __forceinline__ uint4 load_some(const uint4* p, int e0, int e1) {
    const uint16_t* s = reinterpret_cast<const uint16_t*>(p);
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = 2 * i >= e0 && 2 * i < e1 ? s[2 * i] : kNone & 0xffffu;
      const uint32_t hi = 2 * i + 1 >= e0 && 2 * i + 1 < e1 ? s[2 * i + 1] : kNone & 0xffffu;
      x[i] = lo | hi << 16;
    }
    return make_uint4(x[0], x[1], x[2], x[3]);
  }
};
template <>
struct Vec<F32> {
  static constexpr int N = 4;
  static constexpr uint32_t kNone = 0xff800000u;
  static __device__ __forceinline__ void unpack(const uint4& w, float (&f)[4]) {
    f[0] = __uint_as_float(w.x), f[1] = __uint_as_float(w.y), f[2] = __uint_as_float(w.z), f[3] = __uint_as_float(w.w);
  }
  static __device__ __forceinline__ float element(const uint4* p, int i) { return __ldg(reinterpret_cast<const float*>(p) + i); }
  static __device__ __forceinline__ uint4 shifted(const uint4& a, const uint4& b, int by) { return shifted_words(a, b, by); }
  static __device__ __forceinline__ float highest(const uint4& w) {
    return fmaxf(ptx::max3(__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z)), __uint_as_float(w.w));
  }
  static __device__ __forceinline__ float highest(const uint4 (&w)[kPerLane]) {
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i)
      m = ptx::max3(m, ptx::max3(__uint_as_float(w[i].x), __uint_as_float(w[i].y), __uint_as_float(w[i].z)), __uint_as_float(w[i].w));
    return m;
  }
  static __device__ __forceinline__ uint4 load_some(const uint4* p, int e0, int e1) {
    const uint32_t* s = reinterpret_cast<const uint32_t*>(p);
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i >= e0 && i < e1 ? s[i] : kNone;
    return make_uint4(x[0], x[1], x[2], x[3]);
  }
};

// Order-preserving: larger for a larger value; 0 for none.
__device__ __forceinline__ uint32_t order_bits(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);   // (-0 as 0)
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_order_bits(uint32_t b) { return __uint_as_float(b >> 31 ? b ^ 0x80000000u : ~b); }
using Key = unsigned long long;

__device__ __forceinline__ float warp_max(float x) {
  float m;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(x));
  return m;
}

// Whether a beam has continuations from its logits.
__device__ __forceinline__ bool beam_is_live(const BeamLaunch& L, int row) {
  const int ended = L.finished ? __ldg(L.finished + row) : 0;
  const float score = L.scores ? __ldg(L.scores + row) : 0.f;
  return ended == 0 && isfinite(score);
}

// Groups of threads whose maxima bound the n-th largest element.
__device__ __forceinline__ int groups_for(int n) { return n <= 16 ? 64 : n <= 32 ? 128 : 256; }

// A lower bound of the n-th largest of the values whose maxima by thread are `x`:
// the n-th largest of `groups` groups' maxima. The threads of a group share the comparisons. Two barriers.
template <int kBlock>
__device__ __forceinline__ uint32_t bound_of(uint32_t x, uint32_t* group_max, uint32_t* bound, int n, int groups) {
  const int tid = threadIdx.x, width = kBlock / groups, group = tid / width, share = groups / width;
  for (int o = 1; o < width; o <<= 1) x = max(x, __shfl_xor_sync(0xffffffffu, x, o));
  if (tid % width == 0) group_max[group] = x;
  __syncthreads();
  const int first = tid % width * share;
  int rank = 0;
  for (int i = first; i < first + share; i += 8) {
#pragma unroll
    for (int j = i; j < i + 8; ++j) rank += group_max[j] > x || (group_max[j] == x && j < group) ? 1 : 0;
  }
  for (int o = 1; o < width; o <<= 1) rank += __shfl_xor_sync(0xffffffffu, rank, o);
  if (rank == n - 1) *bound = x;
  __syncthreads();
  return *bound;
}

// A block's exponentials are 2^(x kLog2e - c), each exponent rounded once, with c = top kLog2e as it was rounded:
// their sum is in units of 2^(c + top kLog2eLow). Beyond 2^20, where c's rounding would be a large exponent by itself,
// they are 2^((x - top) kLog2e), in units of e^top.
__device__ __forceinline__ bool is_near(float top) { return fabsf(top) < 1048576.f; }
__device__ __forceinline__ float offset_c(float top) { return is_near(top) ? top * kLog2e : 0.f; }

// log2 of the units of (top, c) in units of (to, to_c).
__device__ __forceinline__ float units_between(float top, float c, float to, float to_c) {
  if (is_near(top) && is_near(to)) return fmaf(top - to, kLog2eLow, c - to_c);
  return (top - to) * kLog2e + (is_near(top) ? fmaf(-top, kLog2e, c) : 0.f) - (is_near(to) ? fmaf(-to, kLog2e, to_c) : 0.f);
}

template <class T, bool kFar>
__device__ __forceinline__ float sum_of(const uint4 (&w)[kPerLane], float top, float c) {
  const uint64_t shift = ptx::f2(-top, -top), minus_c = ptx::f2(-c, -c), log2e = ptx::f2(kLog2e, kLog2e);
  uint64_t acc = 0;
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    float x[Vec<T>::N];
    Vec<T>::unpack(w[i], x);
#pragma unroll
    for (int e = 0; e < Vec<T>::N; e += 2) {
      uint64_t y = ptx::f2(x[e], x[e + 1]);
      if constexpr (kFar) y = ptx::add2(y, shift);
      float a, b;
      ptx::unf2(ptx::fma2(y, log2e, minus_c), a, b);
      acc = ptx::add2(acc, ptx::f2(ptx::ex2(a), ptx::ex2(b)));
    }
  }
  float a, b;
  ptx::unf2(acc, a, b);
  return a + b;
}

// A row's vectors of N tokens, -inf beside it. kSkewed: rows may begin inside 16 bytes; a vector is then put together from
// the two that hold it, so that blocks and lanes have the same tokens, and equal rows one sum, wherever they lie.
template <class T, bool kSkewed>
struct Row {
  static constexpr int N = Vec<T>::N;
  const uint4* vectors;             // from the 16 bytes that hold its first element on
  int skew;                         // elements of those before the row
  Row() = default;
  __device__ __forceinline__ Row(const BeamLaunch& L, int b, int k) {
    constexpr int kSize = 16 / N;
    const char* base = static_cast<const char*>(L.logits) + (b * L.ls[0] + k * L.ls[1]) * kSize;
    skew = kSkewed ? static_cast<int>((reinterpret_cast<uintptr_t>(base) & 15) / kSize) : 0;
    vectors = reinterpret_cast<const uint4*>(base - skew * kSize);
  }
  static __device__ __forceinline__ uint4 none() { return make_uint4(Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone); }
  // 16 bytes of memory; what lies beside the row is not read.
  template <bool kOnce>
  __device__ __forceinline__ uint4 aligned(int v, int vocab) const {
    const int before = skew - v * N, after = skew + vocab - v * N;
    if (before <= 0 && after >= N) return kOnce ? load_once(vectors + v) : __ldg(vectors + v);
    return after > 0 ? Vec<T>::load_some(vectors + v, before, after) : none();
  }
  // The chunk at vector `at` as it lies in memory, kSkewed: with the first vector behind it in the first lane; kOnce:
  // nothing of it is read again by this SM.
  static constexpr int kLoads = kPerLane + (kSkewed ? 1 : 0);
  template <bool kOnce>
  __device__ __forceinline__ void load(uint4 (&a)[kLoads], int at, int vocab) const {
    const int lane = threadIdx.x & 31, v = at + lane;
    if ((at + kChunk) * N <= skew + vocab && (at > 0 || skew == 0)) {
#pragma unroll
      for (int i = 0; i < kPerLane; ++i) a[i] = kOnce ? load_once(vectors + v + i * 32) : __ldg(vectors + v + i * 32);
    } else {
#pragma unroll
      for (int i = 0; i < kPerLane; ++i) a[i] = aligned<kOnce>(v + i * 32, vocab);
    }
    if constexpr (kSkewed) a[kPerLane] = lane == 0 ? aligned<kOnce>(at + kChunk, vocab) : none();
  }
  // Its vectors of tokens, by the whole warp.
  __device__ __forceinline__ void put_together(uint4 (&w)[kPerLane], const uint4 (&a)[kLoads]) const {
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
      if constexpr (kSkewed) {
        // The next lane's vector; the last lane's next is the first lane's of the vectors behind.
        const int lane = threadIdx.x & 31, from = (lane + 1) & 31;
        const uint4 give = lane == 0 ? a[i + 1] : a[i];
        const uint4 after = make_uint4(__shfl_sync(0xffffffffu, give.x, from), __shfl_sync(0xffffffffu, give.y, from),
                                       __shfl_sync(0xffffffffu, give.z, from), __shfl_sync(0xffffffffu, give.w, from));
        w[i] = Vec<T>::shifted(a[i], after, skew);
      } else {
        w[i] = a[i];
      }
    }
  }
  __device__ __forceinline__ float element(int token) const { return Vec<T>::element(vectors, token + skew); }
};

// The blocks u, u + L.step, .. below `limit` of all rows' blocks, by a warp. (Counted on without divisions, which
// would cost as much as the exponentials.)
template <class T, bool kSkewed>
__device__ __forceinline__ void scan(const BeamLaunch& L, unsigned u, unsigned limit) {
  const unsigned r = u / L.blocks;
  int j = u - r * L.blocks, b = r / L.beams, k = r - b * L.beams;  // where block u lies
  Row<T, kSkewed> row;
  int at = 0, end = 0;
  // The block, or the next one after it, that is to be read.
  auto advance = [&]() {
    u += L.step;
    j += L.step_block;
    k += L.step_beam;
    b += L.step_batch;
    if (j >= static_cast<int>(L.blocks)) j -= L.blocks, ++k;
    if (k >= L.beams) k -= L.beams, ++b;         // (k was below beams and grew by beams at most)
  };
  auto find = [&]() {
    for (; u < limit; advance()) {
      if (!beam_is_live(L, b * L.beams + k)) continue;
      row = Row<T, kSkewed>(L, b, k);
      at = j * L.block_vectors;
      end = min(at + L.block_vectors, L.row_vectors);
      return true;
    }
    return false;
  };
  uint4 next[Row<T, kSkewed>::kLoads];
  bool more = find();
  if (more) row.template load<true>(next, at, L.vocab);
  float top = -INFINITY, c = 0.f, sum = 0.f, low = 0.f;            // the sum is sum + low
  while (more) {
    uint4 w[kPerLane];
    row.put_together(w, next);
    const unsigned now = u;
    const bool last = at + kChunk >= end;
    if (!last) {
      at += kChunk;
      row.template load<true>(next, at, L.vocab);
    } else {
      advance();
      if ((more = find())) row.template load<true>(next, at, L.vocab);
    }
    const float highest = warp_max(Vec<T>::highest(w));
    if (highest > top) {            // (the whole warp)
      const float to = offset_c(highest);
      if (sum != 0.f) {
        const float f = ptx::ex2(units_between(top, c, highest, to));
        sum *= f, low *= f;
      }
      top = highest, c = to;
    }
    const float add = is_near(top) || top == -INFINITY ? sum_of<T, false>(w, top, c) : sum_of<T, true>(w, top, 0.f);
    const float both = __fadd_rn(sum, add), rest = both - sum;
    low += (sum - (both - rest)) + (add - rest);
    sum = both;
    if (last) {
      sum += low;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if ((threadIdx.x & 31) == 0) L.part[now] = make_float2(top, sum);
      top = -INFINITY, c = 0.f, sum = 0.f, low = 0.f;
    }
  }
}

template <class T, bool kSkewed>
__global__ void __launch_bounds__(kThreads, kPerSm) beam_scan_kernel(const __grid_constant__ BeamLaunch L) {
  ptx::grid_wait();
  ptx::grid_launch_next();
  scan<T, kSkewed>(L, blockIdx.x * kWarps + (threadIdx.x >> 5), L.total);
}

// ---------------------------------------------------------------- the choice
constexpr int kMergeThreads = 512, kMergeWarps = kMergeThreads / 32;
constexpr int kList = 1024;                      // a chunk, at which the threads' maxima may bound nothing
constexpr int kRanked = 160;                     // entries that are ranked by comparing all with all as they are
constexpr int kHeld = 4;                         // blocks of a thread that stay in registers

// A value of 48 bits as the sum of two floats, the second at most half a step of the first.
struct Two {
  float hi, lo;
};
__device__ __forceinline__ Two two_sum(float a, float b) {
  const float s = a + b, t = s - a;
  return {s, (a - (s - t)) + (b - t)};
}
__device__ __forceinline__ Two add(Two a, Two b) {
  const Two s = two_sum(a.hi, b.hi), t = two_sum(a.lo, b.lo);
  Two r = two_sum(s.hi, s.lo + t.hi);
  return two_sum(r.hi, r.lo + t.lo);
}
__device__ __forceinline__ Two add(Two a, float b) {
  const Two s = two_sum(a.hi, b);
  return two_sum(s.hi, s.lo + a.lo);
}

__device__ __forceinline__ Key order_key(Two x) {           // 0: none, beyond the numbers
  return !(fabsf(x.hi) < INFINITY) ? 0 : static_cast<Key>(order_bits(x.hi)) << 32 | order_bits(x.lo);
}
__device__ __forceinline__ float value_of(Key key) {    // the value rounded to fp32
  return key == 0 ? -INFINITY : from_order_bits(static_cast<uint32_t>(key >> 32));
}

constexpr float kLn2 = 0.693147182f, kLn2Low = -1.90465421e-09f;
// ln of s > 0 (s.hi a normal number) times 2^exponent, to about 2^-31: s = 2^e (1 + z + y), 1 + z from 1/sqrt 2 to sqrt 2,
// ln(1 + z + y) = 2 artanh t, t = (z + y) / (2 + z + y), the series from t^3 on and what t's rounding leaves in 32 bits.
__device__ __forceinline__ Two ln(Two s, int exponent) {
  const uint32_t bits = __float_as_uint(s.hi);
  int e = static_cast<int>(bits >> 23) - 127;
  float z = __uint_as_float((bits & 0x7fffffu) | 0x3f800000u) - 1.f;
  float y = s.lo * __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
  if (z > 0.414213562f) z = fmaf(z, 0.5f, -0.5f), y *= 0.5f, ++e;
  const float below = __fadd_rn(2.f, z), by = __frcp_rn(below), cut = z - __fadd_rn(below, -2.f), t = z * by;
  const float left = fmaf(-t, below, z) + fmaf(-t, cut, fmaf(-t, y, y));   // z + y - t (2 + z + y), 2 + z = below + cut
  const float t2 = t * t, rest = fmaf(fmaf(fmaf(fmaf(t2, 2.f / 11.f, 2.f / 9.f), t2, 2.f / 7.f), t2, 0.4f), t2, 2.f / 3.f) * t2 * t;
  const float n = static_cast<float>(e + exponent), q = __fmul_rn(n, kLn2);
  return add(Two{q, fmaf(n, kLn2Low, fmaf(n, kLn2, -q))}, two_sum(2.f * t, fmaf(fmaf(2.f, t2, 2.f) * by, left, rest)));   // (artanh' = 1 + t^2 + ..)
}

// A continuation's place: by value, then by beam, logit and token. A value may leave less of a logit than it has (fp32 logits
// beside a score of -1e9, or near zero), so that the logit decides among equal ones of a beam. (Lists are ranked by it as one number of
// 128 bits, read in one load: 64 sequences of 8 beams over 152,064 tokens take 32.0 us, 33.6 compared key by key.)
struct alignas(16) Place {
  Key rest, value;
  Place() = default;
  __device__ __forceinline__ Place(Key value_, Key rest_) : rest(rest_), value(value_) {}
  __device__ __forceinline__ bool operator>(const Place& o) const { return value > o.value || (value == o.value && rest > o.rest); }
  __device__ __forceinline__ unsigned __int128 number() const { return static_cast<unsigned __int128>(value) << 64 | rest; }
};
__device__ __forceinline__ Key rest_of(int k, float x, int token) {
  return static_cast<Key>(63 - k) << 56 | static_cast<Key>(order_bits(x)) << 24 | static_cast<uint32_t>(0xffffff - token);
}
__device__ __forceinline__ int beam_of(Key rest) { return 63 - static_cast<int>(rest >> 56); }
__device__ __forceinline__ int token_of(Key rest) { return 0xffffff - static_cast<int>(rest & 0xffffff); }

struct MergeShared {
  Two offset[kMaxBeams];                         // score - normaliser; NaN: no continuations from the logits
  float score[kMaxBeams];                        // of a beam that goes on from its logits, else NaN
  float ended_score[kMaxBeams];                  // of a beam that has ended; NaN: it has not, or has none
  Place place[kList];                            // of the listed blocks, then of continuations
  int chosen[kMaxBeamsOut];                      // blocks
  uint32_t group_max[kMergeThreads], bound;
  Place warp_place[kMergeWarps];
  Key least;
  int listed, count;
  uint8_t ended[kMaxBeams];
};

// A row's normaliser in 64 bits, by a warp; NaN: none. (Apart, so that the usual path is short: what a launch of
// a few microseconds spends is also the fetching of its instructions.)
__device__ __noinline__ Two far_normaliser(const float2* part, int blocks) {
  float top = -INFINITY;
  for (int j = threadIdx.x & 31; j < blocks; j += 32) top = fmaxf(top, part[j].x);
  top = warp_max(top);
  double far = 0.0;
  for (int j = threadIdx.x & 31; j < blocks; j += 32) {
    const float2 p = part[j];
    if (p.x == -INFINITY) {
      far += p.y;                   // 0, or not a number
      continue;
    }
    const double c = offset_c(p.x);
    const double from = is_near(p.x) ? 0.693147180559945309417 * (c + static_cast<double>(p.x) * static_cast<double>(kLog2eLow)) : static_cast<double>(p.x);
    far += static_cast<double>(p.y) * exp(from - static_cast<double>(top));
  }
  for (int o = 16; o > 0; o >>= 1) far += __shfl_xor_sync(0xffffffffu, far, o);
  const double x = log(far);
  const float hi = static_cast<float>(x);
  return isfinite(x) && isfinite(top) ? add(two_sum(hi, static_cast<float>(x - static_cast<double>(hi))), top) : Two{NAN, NAN};
}

// A row's normaliser, by a warp; NaN: none. The blocks' sums are added in 48 bits, so that rounding to them is
// not seen beside the blocks' own.
__device__ __forceinline__ Two normaliser(const float2* part, int blocks) {
  constexpr int kBatch = 8;                      // loads on their way at once
  float exponent = -INFINITY;
  Two sum = {0.f, 0.f};                          // the sum is sum 2^exponent
  bool far = false;
  for (int j0 = threadIdx.x & 31; j0 - static_cast<int>(threadIdx.x & 31) < blocks; j0 += kBatch * 32) {
    float2 p[kBatch];
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) p[i] = j0 + i * 32 < blocks ? part[j0 + i * 32] : make_float2(-INFINITY, 0.f);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) top = fmaxf(top, p[i].x), far = far || (!is_near(p[i].x) && p[i].x != -INFINITY);
    top = warp_max(top);
    if (top == -INFINITY) {         // sums of 0, or of what is no number; no exponent yet
#pragma unroll
      for (int i = 0; i < kBatch; ++i) sum.hi += p[i].y;
      continue;
    }
    const float to = fmaxf(exponent, is_near(top) ? ceilf(top * kLog2e) : 0.f);
    const float down = ptx::ex2(exponent - to);
    sum.hi *= down, sum.lo *= down;
    exponent = to;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const float by = p[i].x == -INFINITY ? -INFINITY : fmaf(p[i].x, kLog2eLow, offset_c(p[i].x) - exponent);
      const float f = ptx::ex2(by), product = __fmul_rn(p[i].y, f);
      const Two s = two_sum(sum.hi, product);
      sum.hi = s.hi, sum.lo += s.lo + fmaf(p[i].y, f, -product);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Two s = two_sum(sum.hi, __shfl_xor_sync(0xffffffffu, sum.hi, o));
    sum.hi = s.hi, sum.lo += s.lo + __shfl_xor_sync(0xffffffffu, sum.lo, o);
  }
  if (__any_sync(0xffffffffu, far)) return far_normaliser(part, blocks);
  return sum.hi > 0.f && sum.hi < INFINITY ? ln(two_sum(sum.hi, sum.lo), static_cast<int>(exponent)) : Two{NAN, NAN};
}

// The blocks of a sequence, and the beams that have ended, which are blocks of one.
struct Blocks {
  const BeamLaunch& L;
  const MergeShared& s;
  const float2* part;               // of the sequence
  int b;
  __device__ __forceinline__ int beam(int id) const { return L.blocks == 1 ? id : static_cast<int>(__umulhi(id, L.inverse_blocks)); }
  // What block `id` has at most, its maximum being x.
  __device__ __forceinline__ Key key(int id, float x) const {
    const int k = beam(id);
    const Two offset = s.offset[k];
    if (offset.hi == offset.hi) return x > -INFINITY ? order_key(add(offset, x)) : 0;
    return id == k * static_cast<int>(L.blocks) ? ended(k) : 0;
  }
  // Where its highest continuation stands among those of other blocks: within a beam, blocks are in the order of tokens.
  __device__ __forceinline__ Place place(int id, float x, Key value) const { return {value, rest_of(beam(id), x, id)}; }
  __device__ __forceinline__ Key ended(int k) const {
    const float score = s.ended_score[k];
    return score == score ? order_key({score, 0.f}) : 0;
  }
};

// The chosen blocks' chunks, a warp to each: chunk(beam, row, at, vectors), and ended(beam) of beams that have ended.
template <class T, bool kSkewed, class C, class E>
__device__ __forceinline__ void read_chosen(const Blocks& all, int chosen, C&& chunk, E&& ended) {
  const BeamLaunch& L = all.L;
  const int shift = L.block_shift - kChunkShift;
  for (int u = threadIdx.x >> 5; u < chosen << shift; u += kMergeWarps) {
    const int r = u >> shift, id = all.s.chosen[r], k = all.beam(id);
    if (!(all.s.offset[k].hi == all.s.offset[k].hi)) {
      if ((threadIdx.x & 31) == 0 && u == r << shift) ended(k);
      continue;
    }
    const Row<T, kSkewed> row(L, all.b, k);
    const int at = ((id - k * static_cast<int>(L.blocks)) << L.block_shift) + ((u - (r << shift)) << kChunkShift);
    uint4 w[kPerLane], a[Row<T, kSkewed>::kLoads];
    row.template load<false>(a, at, L.vocab);
    row.put_together(w, a);
    chunk(k, row, at, w);
  }
}

// Their continuations of `least` and above. Vectors that hold one are few: they are found by their maxima and read again.
template <class T, bool kSkewed, class F>
__device__ __forceinline__ void take_chosen(const Blocks& all, int chosen, Key least, F&& take) {
  constexpr int N = Vec<T>::N;
  const float value = value_of(least);
  read_chosen<T, kSkewed>(
      all, chosen,
      [&](int k, const Row<T, kSkewed>& row, int at, const uint4 (&w)[kPerLane]) {
        const Two offset = all.s.offset[k];
        // A logit below this is not of `least`, which the two roundings leave in doubt by less than 2^-22 of either.
        const float lowest = least > 1 ? value - offset.hi - (fabsf(value) + fabsf(offset.hi)) * 0x1p-20f : kLowest;
        unsigned held = 0;
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) held |= Vec<T>::highest(w[i]) >= lowest ? 1u << i : 0u;
        for (; held; held &= held - 1) {
          const int t0 = (at + static_cast<int>(threadIdx.x & 31) + (__ffs(held) - 1) * 32) * N;
          unsigned takes = 0;
#pragma unroll
          for (int e = 0; e < N; ++e) takes |= t0 + e < all.L.vocab && row.element(t0 + e) >= lowest ? 1u << e : 0u;
          for (; takes; takes &= takes - 1) {
            const int t = t0 + __ffs(takes) - 1;
            const float y = row.element(t);
            const Key key = order_key(add(offset, y));
            if (key >= least) take(Place{key, rest_of(k, y, t)});
          }
        }
      },
      [&](int k) {
        const Key key = all.ended(k);
        if (key >= least) take(Place{key, rest_of(k, 0.f, all.L.pad)});
      });
}

// The highest of the CTA's places. (Another barrier before the next call.)
__device__ __forceinline__ Place highest_of(MergeShared& s, Place y) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Place z{__shfl_xor_sync(0xffffffffu, y.value, o), __shfl_xor_sync(0xffffffffu, y.rest, o)};
    if (z > y) y = z;
  }
  if ((threadIdx.x & 31) == 0) s.warp_place[threadIdx.x >> 5] = y;
  __syncthreads();
  for (int i = 0; i < kMergeWarps; ++i) {
    const Place z = s.warp_place[i];
    if (z > y) y = z;
  }
  return y;
}

// What choose() needs of the inputs. (They were there before the scan was: nothing to wait for.)
__device__ __forceinline__ void begin(const BeamLaunch& L, MergeShared& s, int b) {
  if (threadIdx.x == 0) s.count = s.listed = 0;
  for (int k = threadIdx.x; k < L.beams; k += kMergeThreads) {
    const int ended = L.finished ? __ldg(L.finished + b * L.beams + k) : 0;
    const float score = L.scores ? __ldg(L.scores + b * L.beams + k) : 0.f;
    s.score[k] = ended == 0 && isfinite(score) ? score : NAN;
    s.ended_score[k] = ended && isfinite(score) ? score : NAN;
    s.ended[k] = ended ? 1 : 0;
  }
}

// The choice for sequence b, by a CTA, behind begin() and a barrier.
template <class T, bool kSkewed>
__device__ __forceinline__ void choose(const BeamLaunch& L, MergeShared& s, int b) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const Blocks all{L, s, L.part + static_cast<int64_t>(b) * L.beams * L.blocks, b};
  // Each row's normaliser, by a warp; the first blocks' maxima on their way meanwhile.
  const int ids = L.beams * L.blocks;
  float first[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int id = tid + i * kMergeThreads;
    first[i] = id < ids ? all.part[id].x : -INFINITY;              // (of ended beams not used)
  }
  for (int k = warp; k < L.beams; k += kMergeWarps) {
    const float score = s.score[k];
    const Two lse = score == score ? normaliser(all.part + k * static_cast<int64_t>(L.blocks), L.blocks) : Two{NAN, NAN};
    if (lane == 0) s.offset[k] = add({-lse.hi, -lse.lo}, score);
  }
  __syncthreads();

  // The n highest blocks.
  Key held[kHeld], best = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int id = tid + i * kMergeThreads;
    held[i] = id < ids ? all.key(id, first[i]) : 0;
    best = max(best, held[i]);
  }
  for (int id = tid + kHeld * kMergeThreads; id < ids; id += kMergeThreads) best = max(best, all.key(id, all.part[id].x));
  const Key bound = max(static_cast<Key>(bound_of<kMergeThreads>(static_cast<uint32_t>(best >> 32), s.group_max, &s.bound, L.n, groups_for(L.n))) << 32, Key(1));
  if (best >= bound) {
    auto list = [&](int id, float x, Key key) {
      if (key < bound) return;
      const int to = atomicAdd(&s.listed, 1);
      if (to < kList) s.place[to] = all.place(id, x, key);
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i) list(tid + i * kMergeThreads, first[i], held[i]);
    for (int id = tid + kHeld * kMergeThreads; id < ids; id += kMergeThreads) {
      const float x = all.part[id].x;
      list(id, x, all.key(id, x));
    }
  }
  __syncthreads();
  const int listed = s.listed, chosen = min(listed, L.n);
  if (listed <= kList) {
    for (int i = tid; i < listed; i += kMergeThreads) {
      const Place p = s.place[i];
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < listed; ++j) rank += s.place[j].number() > p.number() ? 1 : 0;
      if (rank < L.n) s.chosen[rank] = token_of(p.rest);
      if (rank == L.n - 1) s.least = p.value;
    }
  } else {
    // Many as high as one another: the next one after the last, n times.
    Place last{~Key(0), ~Key(0)};
    for (int r = 0; r < L.n; ++r) {
      Place y{0, 0};
      auto look = [&](int id, float x, Key key) {
        if (key < bound || key > last.value || key < y.value) return;
        const Place p = all.place(id, x, key);
        if (last > p && p > y) y = p;
      };
#pragma unroll
      for (int i = 0; i < kHeld; ++i) look(tid + i * kMergeThreads, first[i], held[i]);
      for (int id = tid + kHeld * kMergeThreads; id < ids; id += kMergeThreads) {
        const float x = all.part[id].x;
        look(id, x, all.key(id, x));
      }
      last = y = highest_of(s, y);
      if (tid == 0) s.chosen[r] = token_of(y.rest), s.least = y.value;
      __syncthreads();
    }
  }
  __syncthreads();

  // Their continuations down to the n-th block's highest; where those are too many, or blocks too few, down to a bound
  // from the continuations themselves.
  Key least = listed >= L.n ? s.least : Key(1);
  for (int tries = listed >= L.n ? 0 : 1;; ++tries) {
    if (tries == 1) {
      best = 0;
      read_chosen<T, kSkewed>(
          all, chosen,
          [&](int k, const Row<T, kSkewed>&, int, const uint4 (&w)[kPerLane]) {
            const float x = Vec<T>::highest(w);
            if (x > -INFINITY) best = max(best, order_key(add(s.offset[k], x)));
          },
          [&](int k) { best = max(best, all.ended(k)); });
      const uint32_t high = bound_of<kMergeThreads>(static_cast<uint32_t>(best >> 32), s.group_max, &s.bound, L.n, kMergeThreads);
      least = max(least, static_cast<Key>(high) << 32);
      if (tid == 0) s.count = 0;
      __syncthreads();
    }
    take_chosen<T, kSkewed>(all, chosen, least, [&](Place p) {
      const int to = atomicAdd(&s.count, 1);
      if (to < kList) s.place[to] = p;
    });
    __syncthreads();
    if (s.count <= kList || tries > 0) break;
    __syncthreads();
  }
  auto put = [&](int rank, Place p) {
    const int64_t to = static_cast<int64_t>(b) * L.n + rank;
    const int k = p.value ? beam_of(p.rest) : -1, v = p.value ? token_of(p.rest) : -1;
    L.score_out[to] = value_of(p.value);
    L.parent[to] = k;
    L.token[to] = v;
    if (L.ended_out) L.ended_out[to] = !p.value || v == L.eos || s.ended[k] ? 1 : 0;
  };
  int count = s.count;
  if (count <= kList) {
    if (count > kRanked) {          // few of them, by a bound from the list itself
      constexpr int kOwn = kList / kMergeThreads;
      Place own[kOwn];
      best = 0;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        const int j = tid + i * kMergeThreads;
        own[i] = j < count ? s.place[j] : Place{0, 0};
        best = max(best, own[i].value);
      }
      const uint32_t high = bound_of<kMergeThreads>(static_cast<uint32_t>(best >> 32), s.group_max, &s.bound, L.n, kMergeThreads);
      if (tid == 0) s.count = 0;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kOwn; ++i)
        if (own[i].value >> 32 >= high && own[i].value > 0) {
          const int to = atomicAdd(&s.count, 1);
          s.place[to] = own[i];
        }
      __syncthreads();
      count = s.count;
    }
    for (int i = tid; i < count; i += kMergeThreads) {
      const Place p = s.place[i];
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < count; ++j) rank += s.place[j].number() > p.number() ? 1 : 0;
      if (rank < L.n) put(rank, p);
    }
    for (int i = count + tid; i < L.n; i += kMergeThreads) put(i, {0, 0});
    return;
  }
  Place last{~Key(0), ~Key(0)};
  for (int r = 0; r < L.n; ++r) {
    Place y{0, 0};
    take_chosen<T, kSkewed>(all, chosen, least, [&](Place p) {
      if (last > p && p > y) y = p;
    });
    last = y = highest_of(s, y);
    if (tid == 0) put(r, y);
    __syncthreads();
  }
}

template <class T, bool kSkewed>
__global__ void __launch_bounds__(kMergeThreads, 2) beam_choice_kernel(const __grid_constant__ BeamLaunch L) {
  __shared__ MergeShared s;
  begin(L, s, blockIdx.x);
  __syncthreads();
  ptx::grid_wait();
  ptx::grid_launch_next();
  choose<T, kSkewed>(L, s, blockIdx.x);
}

// Both for few blocks, at most two to a warp: a cluster per sequence scans its blocks, and its first CTA chooses. The device
// takes as long as for two launches (6.4 us for four beams over 32,000 tokens), the host 4 us less of a call's
// 20; with four blocks a warp the device lost that again (8.6 to 11.9 us for eight beams over 50,264).
template <class T, bool kSkewed>
__global__ void __launch_bounds__(kThreads, kPerSm) beam_small_kernel(const __grid_constant__ BeamLaunch L) {
  static_assert(kThreads == kMergeThreads);
  __shared__ MergeShared s;
  const unsigned rank = ptx::cluster_rank(), b = blockIdx.x / kCluster, first = b * L.beams * L.blocks;
  ptx::grid_wait();
  ptx::grid_launch_next();
  begin(L, s, b);
  scan<T, kSkewed>(L, first + rank * kWarps + (threadIdx.x >> 5), first + L.beams * L.blocks);
  __syncwarp();
  ptx::cluster_sync();              // (the blocks' maxima and sums are seen behind it)
  if (rank == 0) choose<T, kSkewed>(L, s, b);
}

template <class T, bool kSkewed>
cudaError_t launch_both(const BeamLaunch& L, cudaStream_t stream) {
  if (L.small) return launch_clusters(beam_small_kernel<T, kSkewed>, L, L.batch, kThreads, kCluster, stream);
  const cudaError_t e = launch_after(beam_scan_kernel<T, kSkewed>, dim3(L.ctas), kThreads, 0, stream, L);
  return e != cudaSuccess ? e : launch_after(beam_choice_kernel<T, kSkewed>, dim3(L.batch), kMergeThreads, 0, stream, L);
}

template <class T>
cudaError_t launch_t(const BeamLaunch& L, cudaStream_t stream) {
  constexpr int64_t kSize = 16 / Vec<T>::N;
  const bool skewed =
      ((reinterpret_cast<uintptr_t>(L.logits) | (L.batch > 1 ? L.ls[0] * kSize : 0) | (L.beams > 1 ? L.ls[1] * kSize : 0)) & 15) != 0;
  return skewed ? launch_both<T, true>(L, stream) : launch_both<T, false>(L, stream);
}

}  // namespace

BeamSplit beam_split(int64_t rows, int beams, int vocab, int n, int dtype, int n_sm) {
  const int per = dtype == 2 ? 4 : 8;
  BeamSplit s;
  s.row_vectors = (vocab + per - 1) / per;
  // As many bytes of maxima as of chosen blocks to read, within the powers of two: block^2 = 2 beams vocab / n.
  for (s.block_shift = kChunkShift; s.block_shift < 14; ++s.block_shift) {
    const int64_t block = static_cast<int64_t>(per) << s.block_shift;
    if (block * block * n >= 2 * static_cast<int64_t>(beams) * vocab) break;
  }
  s.block_vectors = 1 << s.block_shift;
  s.blocks = (s.row_vectors + s.block_vectors - 1) / s.block_vectors;
  const int64_t most = static_cast<int64_t>(n_sm) * kPerSm;
  s.ctas = static_cast<int>(std::max<int64_t>(1, std::min(most, (rows * s.blocks + kWarps - 1) / kWarps)));
  s.small = static_cast<int64_t>(beams) * s.blocks <= kCluster * kWarps * kSmallBlocks && rows / beams * kCluster <= most;
  s.warps = s.small ? kCluster * kWarps : s.ctas * kWarps;
  return s;
}

cudaError_t launch_beams(const BeamLaunch& L, cudaStream_t stream) {
  return L.dtype == 0 ? launch_t<BF16>(L, stream) : L.dtype == 1 ? launch_t<FP16>(L, stream) : launch_t<F32>(L, stream);
}

}  // namespace evisel
