// How CTAs share the units of a paged-cache call: CTA i of split_ctas() holds the
// units [split_begin(i), split_begin(i + 1)). Plain arithmetic, for kernels and host alike.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define EVISEL_SPLIT_FN __host__ __device__ __forceinline__
#else
#define EVISEL_SPLIT_FN inline
#endif

namespace evisel {

EVISEL_SPLIT_FN int split_min(int a, int b) { return a < b ? a : b; }
EVISEL_SPLIT_FN int split_max(int a, int b) { return a < b ? b : a; }

// CTAs that share `total` units of `problems` problems: each takes at least
// `least`, and where there are many CTAs to a problem their number is a multiple of
// the problems', so that problems of one length are cut at their borders (a
// CTA that crosses one pays its fill and its join twice: 2 us of 10 for one token over 4,160).
// Never more CTAs than units: the join adds up a partial of every CTA between a problem's
// first and last, so that each of them must hold a unit, also where most problems are empty.
EVISEL_SPLIT_FN int split_ctas(int total, int n_ctas, int least, int problems) {
  if (problems * 8 <= n_ctas) {
    const int k = split_min(n_ctas / problems, (total + least * problems - 1) / (least * problems));
    return split_max(1, split_min(total, split_max(1, k) * problems));
  }
  return split_max(1, split_min(n_ctas, (total + least - 1) / least));
}
// CTA i's first unit: floor(i total / ctas), in 32 bits.
EVISEL_SPLIT_FN int split_begin(int i, int total, int ctas) {
  const uint32_t q = static_cast<uint32_t>(total) / ctas, r = static_cast<uint32_t>(total) % ctas;
  return static_cast<int>(i * q + i * r / ctas);     // i, r <= ctas, the CTAs of a grid
}
// The CTA that holds unit u.
EVISEL_SPLIT_FN int split_owner(int u, int total, int ctas) {
  return static_cast<int>((static_cast<int64_t>(u + 1) * ctas - 1) / total);
}

}  // namespace evisel
