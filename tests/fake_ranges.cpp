// Whether bytes hold any of a strided tensor, for the tests.
#include "cache_host.h"

extern "C" int ranges_meet(uint64_t begin, uint64_t end, uint64_t p, int size, int64_t width, int n, const int64_t* sizes,
                           const int64_t* strides) {
  evisel::host::Strided t = {reinterpret_cast<const void*>(p), size, width, n, {}, {}};
  std::copy(sizes, sizes + n, t.sizes);
  std::copy(strides, strides + n, t.strides);
  return evisel::host::meets({static_cast<uintptr_t>(begin), static_cast<uintptr_t>(end)}, t);
}
