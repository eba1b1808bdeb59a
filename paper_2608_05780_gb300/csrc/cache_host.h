// What the host sides of the calls share: argument checks, the scratch of a
// workspace, NVTX ranges. Not part of the public ABI.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>
#include <utility>

#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include "../../include/evisel_cache.h"
#include "cache_internal.h"

namespace evisel {
namespace host {

struct NvtxRange {
  explicit NvtxRange(const char* name) { nvtxRangePushA(name); }
  ~NvtxRange() { nvtxRangePop(); }
  NvtxRange(const NvtxRange&) = delete;
  NvtxRange& operator=(const NvtxRange&) = delete;
};

inline int fail(int code, const std::string& msg) { return set_last_error(code, msg.c_str()); }

inline int cuda_fail(cudaError_t e, const char* what) {
  return fail(EVISEL_ECUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

inline bool misaligned(const void* p, uintptr_t to = 16) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// Bytes [begin, end).
struct Range {
  uintptr_t begin, end;
  bool meets(const Range& o) const { return begin < o.end && o.begin < end; }
};

inline Range range_of(const void* p, int64_t bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(p);
  return {x, x + (p ? static_cast<uintptr_t>(bytes) : 0)};
}

// A strided tensor: runs of `width` elements of `size` bytes, by up to three dimensions (strides in elements, not negative).
struct Strided {
  const void* p;
  int size;
  int64_t width;
  int n;
  int64_t sizes[3], strides[3];
};

// Whether the bytes of `r` hold any of t's own, not of what lies between its runs: in each dimension, outermost
// first, only the first and the last place that reach into r can be there in part. (A dimension inside which another steps further than
// its own step counts as one piece.)
inline bool meets(const Range& r, Strided t) {
  using Wide = __int128;            // strides may be any number
  if (!t.p || r.begin >= r.end || t.width <= 0) return false;
  Wide inner[4] = {static_cast<Wide>(t.width) * t.size};          // bytes of the dimensions inside
  for (int i = 0; i < t.n; ++i) {
    if (t.sizes[i] <= 0) return false;
    if (t.sizes[i] == 1) t.strides[i] = 0;
    for (int j = i; j > 0 && t.strides[j] < t.strides[j - 1]; --j) std::swap(t.strides[j], t.strides[j - 1]), std::swap(t.sizes[j], t.sizes[j - 1]);
  }
  for (int i = 0; i < t.n; ++i) inner[i + 1] = inner[i] + static_cast<Wide>(t.sizes[i] - 1) * t.strides[i] * t.size;
  const auto found = [&](const auto& self, Wide base, int i) -> bool {
    if (base >= r.end || base + inner[i] <= r.begin) return false;
    const Wide step = i > 0 ? static_cast<Wide>(t.strides[i - 1]) * t.size : 0;
    if (i == 0 || base >= r.begin || (step > 0 && step < inner[i - 1])) return true;
    if (step == 0) return self(self, base, i - 1);
    const Wide behind = static_cast<Wide>(r.begin) - base - inner[i - 1], before = static_cast<Wide>(r.end) - base - 1;
    const Wide first = behind < 0 ? 0 : behind / step + 1, last = std::min<Wide>(t.sizes[i - 1] - 1, before / step);
    if (last - first >= 2) return true;
    return first <= last && (self(self, base + first * step, i - 1) || self(self, base + last * step, i - 1));
  };
  return found(found, reinterpret_cast<uintptr_t>(t.p), t.n);
}

// Whether two runs of 32-bit values share any.
inline bool overlap(const int32_t* a, int64_t na, const int32_t* b, int64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + 4 * nb && y < x + 4 * na;
}

constexpr int64_t kMaxStride = int64_t(1) << 38;   // elements: a TMA stride is below 2^40 bytes

inline int check_strides(const int64_t* s, const int64_t* sizes, int n, const char* what) {
  for (int i = 0; i < n; ++i)
    if (sizes[i] > 1 && (s[i] < 0 || s[i] % 8 != 0 || s[i] >= kMaxStride))
      return fail(EVISEL_EINVAL, std::string(what) + " strides must be multiples of 8 elements below 2^38");
  return EVISEL_OK;
}

// A cache's description. `pages`: whether its pages are used at all (an empty batch uses none).
inline int check_cache(const evisel_cache* c, const char* what) {
  if (!c) return fail(EVISEL_EINVAL, std::string(what) + " is NULL");
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(EVISEL_EUNSUPPORTED, "head_dim must be 64 or 128, got " + std::to_string(c->head_dim));
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128)
    return fail(EVISEL_EUNSUPPORTED, "page must be 16, 32, 64 or 128, got " + std::to_string(c->page));
  if (c->dtype != EVISEL_BF16 && c->dtype != EVISEL_FP16) return fail(EVISEL_EUNSUPPORTED, "dtype must be bf16 or fp16");
  if (c->batch < 0 || c->hkv < 1 || c->n_pages < 0 || c->max_pages < 0) return fail(EVISEL_EINVAL, "a size is negative");
  if (c->reserved != 0) return fail(EVISEL_EINVAL, "reserved must be 0");
  if (c->batch > 65535 || c->hkv > 65535 || static_cast<int64_t>(c->batch) * c->hkv > 65535)
    return fail(EVISEL_EUNSUPPORTED, "batch * hkv must be at most 65535");
  if (static_cast<int64_t>(c->max_pages) * c->page > (int64_t(1) << 30))
    return fail(EVISEL_EUNSUPPORTED, "a table row must hold at most 2^30 tokens");
  if (c->batch == 0) return EVISEL_OK;
  if (c->max_pages > 0 && (c->n_pages < 1 || !c->k || !c->v || !c->table))
    return fail(EVISEL_EINVAL, "k, v or table is NULL, or the pool has no page");
  if (!c->lens) return fail(EVISEL_EINVAL, "lens is NULL");
  if (misaligned(c->k) || misaligned(c->v) || misaligned(c->k_mean))
    return fail(EVISEL_EINVAL, "k, v and k_mean must be 16-byte aligned");
  if (misaligned(c->table, 4) || misaligned(c->lens, 4)) return fail(EVISEL_EINVAL, "table and lens must be 4-byte aligned");
  const int64_t sizes[3] = {c->n_pages, c->hkv, c->page};
  for (const int64_t* s : {c->k_stride, c->v_stride})
    for (int i = 0; i < 3; ++i)
      if (sizes[i] > 1 && (s[i] < c->head_dim || s[i] % 8 != 0 || s[i] >= kMaxStride))
        return fail(EVISEL_EINVAL, "page strides must be multiples of 8 elements, from head_dim to below 2^38");
  for (const int64_t* s : {c->table_stride, c->lens_stride})
    if (s[0] < 0 || s[1] < 0) return fail(EVISEL_EINVAL, "table and lens strides must not be negative");
  return EVISEL_OK;
}

inline CacheView view_of(const evisel_cache* c) {
  CacheView v{};
  v.k = c->k;
  v.v = c->v;
  v.k_mean = c->k_mean;
  v.table = c->table;
  v.lens = c->lens;
  std::copy(c->k_stride, c->k_stride + 3, v.ks);
  std::copy(c->v_stride, c->v_stride + 3, v.vs);
  std::copy(c->table_stride, c->table_stride + 2, v.ts);
  std::copy(c->lens_stride, c->lens_stride + 2, v.ls);
  if (c->hkv == 1) v.ls[1] = 0;
  v.batch = c->batch;
  v.hkv = c->hkv;
  v.head_dim = c->head_dim;
  v.page = c->page;
  v.log_page = c->page == 16 ? 4 : c->page == 32 ? 5 : c->page == 64 ? 6 : 7;
  v.n_pages = c->n_pages;
  v.max_pages = c->max_pages;
  v.dtype = c->dtype;
  return v;
}

// Lengths and table that the heads share.
inline Strided lens_of(const evisel_cache* c) { return {c->lens, 4, 1, 1, {c->batch}, {c->lens_stride[0]}}; }
inline Strided table_of(const evisel_cache* c) { return {c->table, 4, c->max_pages, 1, {c->batch}, {c->table_stride[0]}}; }
// The pool's keys or values.
inline Strided pages_of(const evisel_cache* c, const void* p, const int64_t* stride) {
  return {p, 2, c->head_dim, 3, {c->n_pages, c->hkv, c->page}, {stride[0], stride[1], stride[2]}};
}

// What an append needs of its arguments.
inline int check_append(const evisel_cache* cache, const evisel_draft* draft, const int32_t* src, const int32_t* counts,
                        const int32_t* lens_out, evisel_ws** ws_inout) {
  int rc = check_cache(cache, "cache");
  if (rc != EVISEL_OK) return rc;
  if (!draft) return fail(EVISEL_EINVAL, "draft is NULL");
  if (!ws_inout) return fail(EVISEL_EINVAL, "ws_inout is NULL");
  if (draft->tokens < 0) return fail(EVISEL_EINVAL, "tokens is negative");
  if (draft->tokens > (1 << 30)) return fail(EVISEL_EUNSUPPORTED, "tokens must be at most 2^30");
  if (draft->reserved != 0) return fail(EVISEL_EINVAL, "reserved must be 0");
  if (cache->hkv > 1 && (cache->table_stride[1] != 0 || cache->lens_stride[1] != 0))
    return fail(EVISEL_EUNSUPPORTED, "an append needs a table and lengths that the heads share");
  if (cache->batch == 0) return EVISEL_OK;
  if (!lens_out || lens_out == cache->lens) return fail(EVISEL_EINVAL, "lens_out is NULL or the cache's lens");
  if (misaligned(lens_out, 4) || misaligned(src, 4) || misaligned(counts, 4))
    return fail(EVISEL_EINVAL, "src, counts and lens_out must be 4-byte aligned");
  if (overlap(lens_out, cache->batch, counts, cache->batch) ||
      overlap(lens_out, cache->batch, src, static_cast<int64_t>(cache->batch) * draft->tokens))
    return fail(EVISEL_EINVAL, "lens_out must not overlap counts or src");
  // Other blocks still read the lengths.
  if (meets(range_of(lens_out, 4 * static_cast<int64_t>(cache->batch)), lens_of(cache)))
    return fail(EVISEL_EINVAL, "lens_out must not overlap the cache's lens");
  if (draft->tokens > 0) {
    if (!draft->k_new || !draft->v_new) return fail(EVISEL_EINVAL, "k_new or v_new is NULL");
    if (misaligned(draft->k_new) || misaligned(draft->v_new)) return fail(EVISEL_EINVAL, "k_new and v_new must be 16-byte aligned");
    const int64_t sizes[3] = {cache->batch, draft->tokens, cache->hkv};
    rc = check_strides(draft->k_new_stride, sizes, 3, "k_new");
    if (rc == EVISEL_OK) rc = check_strides(draft->v_new_stride, sizes, 3, "v_new");
    if (rc != EVISEL_OK) return rc;
  }
  return EVISEL_OK;
}

inline CacheAppendLaunch append_of(const evisel_cache* cache, const evisel_draft* draft, const int32_t* src,
                                   const int32_t* counts, int32_t* lens_out, evisel_ws* ws) {
  CacheAppendLaunch L{};
  L.c = view_of(cache);
  L.d.tokens = draft->tokens;
  L.d.k_new = draft->k_new;
  L.d.v_new = draft->v_new;
  std::copy(draft->k_new_stride, draft->k_new_stride + 3, L.d.kns);
  std::copy(draft->v_new_stride, draft->v_new_stride + 3, L.d.vns);
  L.src = src;
  L.counts = counts;
  L.lens_out = lens_out;
  L.status = ws_status(ws);
  return L;
}

// Whether a call on `stream` may allocate now.
inline int check_may_allocate(cudaStream_t stream, const char* what) {
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  const cudaError_t e = cudaStreamIsCapturing(stream, &capture);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return cuda_fail(e, "cudaStreamIsCapturing");
  }
  if (capture != cudaStreamCaptureStatusNone)
    return fail(EVISEL_EINVAL, std::string(what) + " during a stream capture: make a call of this size before it, on the same workspace");
  return EVISEL_OK;
}

// The caller's workspace, or a new one.
inline int acquire(evisel_ws** ws_inout, cudaStream_t stream) {
  if (!*ws_inout) {
    const int rc = check_may_allocate(stream, "a workspace cannot be created");
    if (rc != EVISEL_OK) return rc;
  }
  return ws_acquire(ws_inout);
}

// Scratch of `need` bytes. A smaller one stays until the workspace is freed: captured
// graphs, and calls in flight, hold its address. Each is at least half as large again
// as the one before it, so that all of them together are at most 4.5 times the largest need.
inline int grow(evisel_ws* ws, size_t need, cudaStream_t stream) {
  WsCache& w = ws_cache(ws);
  if (need <= w.bytes) return EVISEL_OK;
  const int rc = check_may_allocate(stream, "the workspace cannot grow");
  if (rc != EVISEL_OK) return rc;
  const size_t bytes = std::max(need, w.bytes + w.bytes / 2);
  w.outgrown.reserve(w.outgrown.size() + 1);     // (what may throw, before the allocation)
  void* buf = nullptr;
  if (cudaMalloc(&buf, bytes) != cudaSuccess) {
    cudaGetLastError();
    return fail(EVISEL_ENOMEM, "cache scratch of " + std::to_string(bytes) + " bytes");
  }
  if (w.buf) w.outgrown.push_back(w.buf);
  w.buf = buf;
  w.bytes = bytes;
  w.held += bytes;
  return EVISEL_OK;
}

// One call: its NVTX range, and no exception past the C boundary.
template <class F>
int guarded(const char* name, F&& call) {
  const NvtxRange range(name);
  try {
    clear_last_error();
    return call();
  } catch (...) {                   // host memory for a message or a workspace
    return EVISEL_ENOMEM;
  }
}

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

}  // namespace host
}  // namespace evisel
