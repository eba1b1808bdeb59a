// Host side of the paged-cache calls (evisel_cache.h): argument checks, scratch
// of the workspace, TMA descriptors and kernel launches.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include <cuda_runtime.h>

#include "cache_host.h"

using namespace evisel;
using namespace evisel::host;

namespace {

constexpr int kMaxDrafted = 1024;
constexpr int kMaxGroup = 128;
constexpr int kMaxSelectPages = 8192;
constexpr int64_t kMaxUnits = int64_t(1) << 30;    // of work in a call: the kernels count them in 32 bits

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
    int rc = check_append(cache, draft, src, counts, lens_out, ws_inout);
    if (rc != EVISEL_OK || cache->batch == 0) return rc;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    rc = acquire(ws_inout, stream);
    if (rc != EVISEL_OK) return rc;
    const CacheAppendLaunch L = append_of(cache, draft, src, counts, lens_out, *ws_inout);
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
