// Host side of the paged-cache calls (evisel_cache.h): argument checks, scratch
// of the workspace, TMA descriptors and kernel launches.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include "../../include/evisel_cache.h"
#include "cache_internal.h"

using namespace evisel;

namespace {

struct NvtxRange {
  explicit NvtxRange(const char* name) { nvtxRangePushA(name); }
  ~NvtxRange() { nvtxRangePop(); }
  NvtxRange(const NvtxRange&) = delete;
  NvtxRange& operator=(const NvtxRange&) = delete;
};

int fail(int code, const std::string& msg) { return set_last_error(code, msg.c_str()); }

int cuda_fail(cudaError_t e, const char* what) {
  return fail(EVISEL_ECUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

bool misaligned(const void* p, uintptr_t to = 16) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// Whether two runs of 32-bit values share any.
bool overlap(const int32_t* a, int64_t na, const int32_t* b, int64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + 4 * nb && y < x + 4 * na;
}

constexpr int64_t kMaxStride = int64_t(1) << 38;   // elements: a TMA stride is below 2^40 bytes
constexpr int kMaxDrafted = 1024;
constexpr int kMaxGroup = 128;
constexpr int kMaxSelectPages = 8192;
constexpr int64_t kMaxUnits = int64_t(1) << 30;    // of work in a call: the kernels count them in 32 bits

int check_strides(const int64_t* s, const int64_t* sizes, int n, const char* what) {
  for (int i = 0; i < n; ++i)
    if (sizes[i] > 1 && (s[i] < 0 || s[i] % 8 != 0 || s[i] >= kMaxStride))
      return fail(EVISEL_EINVAL, std::string(what) + " strides must be multiples of 8 elements below 2^38");
  return EVISEL_OK;
}

// A cache's description. `pages`: whether its pages are used at all (an empty batch uses none).
int check_cache(const evisel_cache* c, const char* what) {
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

int check_draft(const evisel_cache* c, const evisel_draft* d, bool new_tokens) {
  if (!d) return fail(EVISEL_EINVAL, "draft is NULL");
  if (d->tokens < 0) return fail(EVISEL_EINVAL, "tokens is negative");
  if (d->tokens > kMaxDrafted) return fail(EVISEL_EUNSUPPORTED, "tokens must be at most " + std::to_string(kMaxDrafted));
  if (d->hq < 1 || d->hq % c->hkv != 0) return fail(EVISEL_EUNSUPPORTED, "hq must be a multiple of hkv");
  if (d->hq / c->hkv > kMaxGroup) return fail(EVISEL_EUNSUPPORTED, "hq / hkv must be at most " + std::to_string(kMaxGroup));
  if (!(d->softmax_scale >= 0.f) || !std::isfinite(d->softmax_scale))
    return fail(EVISEL_EINVAL, "softmax_scale must be finite and >= 0");
  if (d->reserved != 0) return fail(EVISEL_EINVAL, "reserved must be 0");
  if (c->batch == 0 || d->tokens == 0) return EVISEL_OK;
  if (!d->q) return fail(EVISEL_EINVAL, "q is NULL");
  if (misaligned(d->q)) return fail(EVISEL_EINVAL, "q must be 16-byte aligned");
  const int64_t q_sizes[3] = {c->batch, d->tokens, d->hq}, kv_sizes[3] = {c->batch, d->tokens, c->hkv};
  int rc = check_strides(d->q_stride, q_sizes, 3, "q");
  if (rc != EVISEL_OK) return rc;
  if (misaligned(d->drafted, 4)) return fail(EVISEL_EINVAL, "drafted must be 4-byte aligned");
  if (!new_tokens || !d->k_new) return EVISEL_OK;
  if (!d->v_new) return fail(EVISEL_EINVAL, "k_new without v_new");
  if (misaligned(d->k_new) || misaligned(d->v_new)) return fail(EVISEL_EINVAL, "k_new and v_new must be 16-byte aligned");
  rc = check_strides(d->k_new_stride, kv_sizes, 3, "k_new");
  if (rc == EVISEL_OK) rc = check_strides(d->v_new_stride, kv_sizes, 3, "v_new");
  if (rc != EVISEL_OK) return rc;
  if (d->tree && (misaligned(d->tree, 4) || d->tree_stride[0] < 0 || d->tree_stride[1] < 0))
    return fail(EVISEL_EINVAL, "tree must be 4-byte aligned, its strides not negative");
  return EVISEL_OK;
}

CacheView view_of(const evisel_cache* c) {
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

DraftView view_of(const evisel_cache* c, const evisel_draft* d) {
  DraftView v{};
  v.q = d->q;
  v.k_new = d->k_new;
  v.v_new = d->v_new;
  v.tree = d->tree;
  v.drafted = d->drafted;
  std::copy(d->q_stride, d->q_stride + 3, v.qs);
  std::copy(d->k_new_stride, d->k_new_stride + 3, v.kns);
  std::copy(d->v_new_stride, d->v_new_stride + 3, v.vns);
  std::copy(d->tree_stride, d->tree_stride + 2, v.trs);
  v.tokens = d->tokens;
  v.hq = d->hq;
  v.gq = d->hq / c->hkv;
  const float scale = d->softmax_scale > 0.f ? d->softmax_scale : 1.0f / std::sqrt(static_cast<float>(c->head_dim));
  v.scale_log2 = scale * 1.4426950408889634f;
  return v;
}

// 4-D map {d, ...} of a tensor whose other dimensions are token, head and page (or
// sequence), placed in the order of their strides (a dimension of one entry
// takes any); `perm` gets the place, 1..3, of each: two bits, in that order.
struct MapDim {
  int64_t stride;                   // elements
  int64_t size;
  int box;
};

int encode_sorted(CUtensorMap* map, int* perm, const void* base, int head_dim, int dtype, const MapDim (&in)[3]) {
  struct {
    MapDim x;
    int what;
  } dim[3] = {{in[0], 0}, {in[1], 1}, {in[2], 2}};
  for (auto& d : dim)
    if (d.x.size == 1) d.x.stride = head_dim;
  std::stable_sort(dim, dim + 3, [](const auto& a, const auto& b) { return a.x.stride < b.x.stride; });
  uint64_t dims[4] = {static_cast<uint64_t>(head_dim)}, strides[3];
  uint32_t box[4] = {64u};
  *perm = 0;
  for (int i = 0; i < 3; ++i) {
    dims[i + 1] = static_cast<uint64_t>(dim[i].x.size);
    strides[i] = static_cast<uint64_t>(dim[i].x.stride) * 2;
    box[i + 1] = static_cast<uint32_t>(dim[i].x.box);
    *perm |= (i + 1) << (2 * dim[i].what);
  }
  return encode_map4(map, base, dtype, dims, strides, box);
}

// The pages of k or v, box of box_rows tokens of one page and head.
int encode_pages(CUtensorMap* map, int* perm, const void* base, const evisel_cache* c, const int64_t* stride, int box_rows) {
  return encode_sorted(map, perm, base, c->head_dim, c->dtype,
                       {{stride[2], c->page, box_rows}, {stride[1], c->hkv, 1}, {stride[0], c->n_pages, 1}});
}

// Whether a TMA map can describe q: no repeated (stride 0) dimension.
bool has_query_map(const evisel_cache* c, const evisel_draft* d) {
  const int64_t sizes[3] = {c->batch, d->tokens, d->hq};
  for (int i = 0; i < 3; ++i)
    if (sizes[i] > 1 && d->q_stride[i] == 0) return false;
  return true;
}

// The tokens cut evenly into as few tiles of at most 128 rows as hold them.
QueryTile query_tile(const evisel_cache* c, const evisel_draft* d) {
  const int gq = d->hq / c->hkv, most = 128 / gq;
  QueryTile t{};
  const int tiles = std::max(1, (d->tokens + most - 1) / most);
  t.tokens = std::max(1, (d->tokens + tiles - 1) / tiles);
  t.rows = t.tokens * gq;
  return t;
}

// The queries, box of a tile. The rows follow the order of the strides.
int encode_queries(CUtensorMap* map, int* perm, QueryTile* tile, const evisel_cache* c, const evisel_draft* d) {
  const int rc = encode_sorted(map, perm, d->q, c->head_dim, c->dtype,
                               {{d->q_stride[1], d->tokens, tile->tokens}, {d->q_stride[2], d->hq, d->hq / c->hkv},
                                {d->q_stride[0], c->batch, 1}});
  tile->head_inner = ((*perm >> 2) & 3) < (*perm & 3);
  return rc;
}

// Whether a call on `stream` may allocate now.
int check_may_allocate(cudaStream_t stream, const char* what) {
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
int acquire(evisel_ws** ws_inout, cudaStream_t stream) {
  if (!*ws_inout) {
    const int rc = check_may_allocate(stream, "a workspace cannot be created");
    if (rc != EVISEL_OK) return rc;
  }
  return ws_acquire(ws_inout);
}

// Scratch of `need` bytes. A smaller one stays until the workspace is freed: captured
// graphs, and calls in flight, hold its address. Each is at least half as large again
// as the one before it, so that all of them together are at most 4.5 times the largest need.
int grow(evisel_ws* ws, size_t need, cudaStream_t stream) {
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

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

}  // namespace

extern "C" {

int evisel_cache_attention(const evisel_cache* cache, const evisel_draft* draft, void* o, float* lse, void* stream_ptr,
                           evisel_ws** ws_inout) {
  return guarded("evisel_cache_attention", [&]() -> int {
    int rc = check_cache(cache, "cache");
    if (rc == EVISEL_OK) rc = check_draft(cache, draft, true);
    if (rc != EVISEL_OK) return rc;
    if (!ws_inout) return fail(EVISEL_EINVAL, "ws_inout is NULL");
    if (cache->batch == 0 || draft->tokens == 0) return EVISEL_OK;
    if (!o || !lse) return fail(EVISEL_EINVAL, "o or lse is NULL");
    if (misaligned(o) || misaligned(lse, 4)) return fail(EVISEL_EINVAL, "o must be 16-byte aligned, lse 4-byte");
    const int n_sm = sm_count();
    if (n_sm <= 0) return fail(EVISEL_ECUDA, "the device's multiprocessors cannot be counted");

    CacheAttnLaunch L{};
    L.c = view_of(cache);
    L.d = view_of(cache, draft);
    L.rows = draft->tokens * L.d.gq;
    L.qt = query_tile(cache, draft);
    const int64_t capacity = static_cast<int64_t>(cache->max_pages) * cache->page;
    const CacheAttnShape shape = cache_attn_shape(L.rows, draft->tokens, static_cast<int64_t>(cache->batch) * cache->hkv, capacity,
                                                  cache->head_dim, L.qt, has_query_map(cache, draft), n_sm);
    L.wide = shape.wide;
    L.slots = shape.slots;
    L.slot_rows = shape.slot_rows;
    L.tile_rows = shape.tile_rows;
    L.row_tiles = shape.row_tiles;
    L.key_tile = shape.key_tile;
    L.n_ctas = shape.n_ctas;
    L.min_units = shape.min_units;
    L.lead = shape.lead;
    L.join_tile = shape.join_tile;
    L.join_warps = shape.join_warps;
    L.box_rows = std::min(cache->page, L.key_tile);
    const int64_t problems = static_cast<int64_t>(cache->batch) * cache->hkv * L.row_tiles;
    const int64_t tiles = (capacity + L.key_tile - 1) / L.key_tile;
    if (problems * (tiles + L.lead) > kMaxUnits) return fail(EVISEL_EUNSUPPORTED, "too many units of work");
    const size_t parts = static_cast<size_t>(L.n_ctas) + problems;
    const size_t ml_bytes = align_up(parts * L.tile_rows * sizeof(float2), 256);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    rc = acquire(ws_inout, stream);
    if (rc == EVISEL_OK) rc = grow(*ws_inout, ml_bytes + parts * L.tile_rows * cache->head_dim * sizeof(float), stream);
    if (rc == EVISEL_OK && cache->max_pages > 0) rc = encode_pages(&L.tm_k, &L.k_perm, cache->k, cache, cache->k_stride, L.box_rows);
    if (rc == EVISEL_OK && cache->max_pages > 0) rc = encode_pages(&L.tm_v, &L.v_perm, cache->v, cache, cache->v_stride, L.box_rows);
    if (rc == EVISEL_OK && L.wide) rc = encode_queries(&L.tm_q, &L.q_perm, &L.qt, cache, draft);
    if (rc != EVISEL_OK) return rc;
    char* buf = static_cast<char*>(ws_cache(*ws_inout).buf);
    L.part_ml = reinterpret_cast<float2*>(buf);
    L.part_o = reinterpret_cast<float*>(buf + ml_bytes);
    L.o = o;
    L.lse = lse;
    L.status = ws_status(*ws_inout);
    const cudaError_t e = launch_cache_attn(L, stream);
    if (e != cudaSuccess) return cuda_fail(e, "cache attention launch");
    ws_ran_on(*ws_inout, stream);
    return EVISEL_OK;
  });
}

int evisel_cache_evidence(const evisel_cache* cache, const evisel_draft* draft, const float* lse, const uint8_t* use,
                          float* acc, int64_t acc_len, int accumulate, void* stream_ptr, evisel_ws** ws_inout) {
  return guarded("evisel_cache_evidence", [&]() -> int {
    int rc = check_cache(cache, "cache");
    if (rc == EVISEL_OK) rc = check_draft(cache, draft, false);
    if (rc != EVISEL_OK) return rc;
    if (!ws_inout) return fail(EVISEL_EINVAL, "ws_inout is NULL");
    if (acc_len < 0) return fail(EVISEL_EINVAL, "acc_len is negative");
    if (cache->batch == 0 || cache->max_pages == 0) return EVISEL_OK;
    if ((acc_len > 0 && !acc) || (draft->tokens > 0 && !lse)) return fail(EVISEL_EINVAL, "acc or lse is NULL");
    if (misaligned(acc, 4) || misaligned(lse, 4)) return fail(EVISEL_EINVAL, "acc and lse must be 4-byte aligned");
    CacheEvidenceLaunch L{};
    L.c = view_of(cache);
    L.d = view_of(cache, draft);
    L.n_ctas = sm_count();
    if (L.n_ctas <= 0) return fail(EVISEL_ECUDA, "the device's multiprocessors cannot be counted");
    L.box_rows = std::min(cache->page, 128);
    L.qt = query_tile(cache, draft);
    L.has_q_map = draft->tokens > 0 && has_query_map(cache, draft);
    if (static_cast<int64_t>(cache->batch) * cache->hkv * ((static_cast<int64_t>(cache->max_pages) * cache->page + 127) / 128) > kMaxUnits)
      return fail(EVISEL_EUNSUPPORTED, "too many units of work");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    rc = acquire(ws_inout, stream);
    if (rc == EVISEL_OK && L.has_q_map) rc = encode_pages(&L.tm_k, &L.k_perm, cache->k, cache, cache->k_stride, L.box_rows);
    if (rc == EVISEL_OK && L.has_q_map) rc = encode_queries(&L.tm_q, &L.q_perm, &L.qt, cache, draft);
    if (rc != EVISEL_OK) return rc;
    L.lse = lse;
    L.use = use;
    L.acc = acc;
    L.acc_len = acc_len;
    L.status = ws_status(*ws_inout);
    L.accumulate = accumulate != 0;
    const cudaError_t e = launch_cache_evidence(L, stream);
    if (e != cudaSuccess) return cuda_fail(e, "cache evidence launch");
    ws_ran_on(*ws_inout, stream);
    return EVISEL_OK;
  });
}

int evisel_cache_evict(const evisel_cache* cache, const float* acc, int64_t acc_len, const evisel_cache* out,
                       int32_t budget, int32_t sink, int32_t recent, int32_t* kept, float* acc_out,
                       int64_t acc_out_len, void* stream_ptr, evisel_ws** ws_inout) {
  return guarded("evisel_cache_evict", [&]() -> int {
    int rc = check_cache(cache, "cache");
    if (rc == EVISEL_OK) rc = check_cache(out, "out");
    if (rc != EVISEL_OK) return rc;
    if (!ws_inout) return fail(EVISEL_EINVAL, "ws_inout is NULL");
    if (out->batch != cache->batch || out->hkv != cache->hkv || out->head_dim != cache->head_dim || out->dtype != cache->dtype)
      return fail(EVISEL_EINVAL, "out must have the cache's batch, heads, head_dim and dtype");
    if (budget < 1 || sink < 0 || recent < 0 || static_cast<int64_t>(sink) + recent > budget)
      return fail(EVISEL_EINVAL, "budget must be at least 1 and hold sink and recent");
    if (static_cast<int64_t>(out->max_pages) * out->page < budget) return fail(EVISEL_EINVAL, "out has no room for budget tokens");
    if (acc_len < 0 || acc_out_len < budget) return fail(EVISEL_EINVAL, "acc_len is negative, or acc_out_len below budget");
    if (cache->batch == 0) return EVISEL_OK;
    if (cache->hkv > 1 && cache->lens_stride[1] != 0 && out->lens_stride[1] == 0)
      return fail(EVISEL_EINVAL, "lengths per head need lengths per head in out");
    if ((acc_len > 0 && !acc) || !kept || !acc_out) return fail(EVISEL_EINVAL, "acc, kept or acc_out is NULL");
    if (misaligned(acc, 4) || misaligned(kept, 4) || misaligned(acc_out, 4))
      return fail(EVISEL_EINVAL, "acc, kept and acc_out must be 4-byte aligned");
    if (acc == acc_out || out->lens == cache->lens || (out->k == cache->k && out->table == cache->table))
      return fail(EVISEL_EINVAL, "out and acc_out must not be the cache's own");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    rc = acquire(ws_inout, stream);
    if (rc != EVISEL_OK) return rc;
    CacheEvictLaunch L{};
    L.c = view_of(cache);
    L.out = view_of(out);
    L.out_k = out->k;
    L.out_v = out->v;
    L.out_mean = out->k_mean;
    L.out_lens = out->lens;
    L.acc = acc;
    L.acc_len = acc_len;
    L.kept = kept;
    L.acc_out = acc_out;
    L.acc_out_len = acc_out_len;
    L.budget = budget;
    L.sink = sink;
    L.recent = recent;
    L.status = ws_status(*ws_inout);
    const cudaError_t e = launch_cache_evict(L, stream);
    if (e != cudaSuccess) return cuda_fail(e, "cache eviction launch");
    ws_ran_on(*ws_inout, stream);
    return EVISEL_OK;
  });
}

int evisel_cache_append(const evisel_cache* cache, const evisel_draft* draft, const int32_t* src, const int32_t* counts,
                        int32_t* lens_out, void* stream_ptr, evisel_ws** ws_inout) {
  return guarded("evisel_cache_append", [&]() -> int {
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
    if (draft->tokens > 0) {
      if (!draft->k_new || !draft->v_new) return fail(EVISEL_EINVAL, "k_new or v_new is NULL");
      if (misaligned(draft->k_new) || misaligned(draft->v_new)) return fail(EVISEL_EINVAL, "k_new and v_new must be 16-byte aligned");
      const int64_t sizes[3] = {cache->batch, draft->tokens, cache->hkv};
      rc = check_strides(draft->k_new_stride, sizes, 3, "k_new");
      if (rc == EVISEL_OK) rc = check_strides(draft->v_new_stride, sizes, 3, "v_new");
      if (rc != EVISEL_OK) return rc;
    }
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    rc = acquire(ws_inout, stream);
    if (rc != EVISEL_OK) return rc;
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
    L.status = ws_status(*ws_inout);
    const cudaError_t e = launch_cache_append(L, stream);
    if (e != cudaSuccess) return cuda_fail(e, "cache append launch");
    ws_ran_on(*ws_inout, stream);
    return EVISEL_OK;
  });
}

int evisel_cache_select(const evisel_cache* cache, const evisel_draft* draft, int32_t n_select, int32_t sink,
                        int32_t recent, int32_t* pages, int32_t* sel_table, int32_t* sel_lens, void* stream_ptr,
                        evisel_ws** ws_inout) {
  return guarded("evisel_cache_select", [&]() -> int {
    int rc = check_cache(cache, "cache");
    if (rc == EVISEL_OK) rc = check_draft(cache, draft, false);
    if (rc != EVISEL_OK) return rc;
    if (!ws_inout) return fail(EVISEL_EINVAL, "ws_inout is NULL");
    if (sink < 0 || recent < 1 || static_cast<int64_t>(sink) + recent > n_select)
      return fail(EVISEL_EINVAL, "n_select must hold sink >= 0 and recent >= 1");
    if (cache->max_pages > kMaxSelectPages)
      return fail(EVISEL_EUNSUPPORTED, "max_pages must be at most " + std::to_string(kMaxSelectPages));
    if (cache->batch == 0) return EVISEL_OK;
    if (!pages || !sel_table || !sel_lens) return fail(EVISEL_EINVAL, "an output is NULL");
    if (misaligned(pages, 4) || misaligned(sel_table, 4) || misaligned(sel_lens, 4))
      return fail(EVISEL_EINVAL, "outputs must be 4-byte aligned");
    if (cache->max_pages > 0 && !cache->k_mean) return fail(EVISEL_EINVAL, "the cache has no k_mean");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    rc = acquire(ws_inout, stream);
    if (rc != EVISEL_OK) return rc;
    CacheSelectLaunch L{};
    L.c = view_of(cache);
    L.d = view_of(cache, draft);
    L.pages = pages;
    L.sel_table = sel_table;
    L.sel_lens = sel_lens;
    L.n_select = n_select;
    L.sink = sink;
    L.recent = recent;
    L.status = ws_status(*ws_inout);
    const cudaError_t e = launch_cache_select(L, stream);
    if (e != cudaSuccess) return cuda_fail(e, "cache selection launch");
    ws_ran_on(*ws_inout, stream);
    return EVISEL_OK;
  });
}

}  // extern "C"
