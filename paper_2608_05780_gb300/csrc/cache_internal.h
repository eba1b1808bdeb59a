// Structures shared by the host side of the paged-cache calls (evisel_cache.cpp)
// and their kernels. Not part of the public ABI.
#pragma once

#include <vector>

#include "evisel_internal.h"

struct evisel_ws;

namespace evisel {

// A cache as the kernels read it. Lengths and page ids are device memory, so
// every use is checked there: see cache_len() and cache_page().
struct CacheView {
  const void* k;
  const void* v;
  const void* k_mean;               // [n_pages, hkv, d] or null
  const int32_t* table;
  const int32_t* lens;
  int64_t ks[3], vs[3];             // page, head, token (elements)
  int64_t ts[2], ls[2];             // sequence, head
  int batch, hkv, head_dim, page, log_page, n_pages, max_pages, dtype;
};

// One call's drafted tokens (rows r = token * gq + head of the group).
struct DraftView {
  const void* q;
  const void* k_new;                // or null
  const void* v_new;
  const int32_t* tree;              // or null: a chain
  const int32_t* drafted;           // or null: all
  int64_t qs[3], kns[3], vns[3];    // sequence, token, head (elements)
  int64_t trs[2];                   // sequence, token
  int tokens, hq, gq;
  float scale_log2;                 // softmax_scale * log2(e)
};

// Rows of a tile of queries of one (sequence, KV head), as their map's box lays
// them out: all gq heads of `tokens` tokens, the heads inside a token's rows or
// the tokens inside a head's.
struct QueryTile {
  int tokens, rows;                 // rows = tokens * gq <= 128
  int head_inner;
};

// Attention: the cached keys of every (sequence, KV head, tile of tile_rows
// rows), a problem, are cut into units of key_tile keys; `lead` units without keys
// stand before them. All units are dealt evenly over n_ctas CTAs in order. A
// CTA's part of a problem leaves a partial: the one of CTA i and problem p is
// partial i + p (both never fall along the units, so no two are the same).
struct CacheAttnLaunch {
  CUtensorMap tm_k, tm_v;           // pages; box {64, box_rows, 1, 1} in the order of `perm`
  CUtensorMap tm_q;                 // wide: queries, box of gq heads of tile_tokens tokens
  CacheView c;
  DraftView d;
  void* o;
  float* lse;
  float* part_o;                    // [partials, tile_rows, d], unnormalised
  float2* part_ml;                  // [partials, tile_rows]: running max (log2 units, less T::kHeadroom), row sum
  int* status;
  int k_perm, v_perm, q_perm;       // where token, head and page (sequence) stand in the maps' coordinates
  int box_rows;
  int rows, tile_rows, row_tiles;   // rows = tokens * gq; tile_rows rows of a partial
  int slots, slot_rows;             // a row tile is `slots` slots of slot_rows rows, tile_rows / slots places each
  QueryTile qt;                     // wide: the rows of a slot
  int n_ctas, key_tile;
  int min_units;                    // that a CTA takes at least
  int lead;                         // units that stand for a problem's fill and join
  int join_tile, join_warps;        // join by tiles of 16 rows or row by row; the warps (1, 2, 4, 8) that share one
  int wide;                         // 128-row slots on tcgen05 (else mma.sync)
};

struct CacheEvidenceLaunch {
  CUtensorMap tm_k, tm_q;           // pages, queries
  CacheView c;
  DraftView d;
  QueryTile qt;
  int has_q_map;                    // tm_q and qt describe q
  const float* lse;                 // [hq, B, T]
  const uint8_t* use;               // [B, T] or null
  float* acc;                       // [B, hkv, acc_len]
  int64_t acc_len;
  int* status;
  int k_perm, q_perm, box_rows, n_ctas;
  int accumulate;
};

struct CacheEvictLaunch {
  CacheView c, out;
  void* out_k;
  void* out_v;
  void* out_mean;
  int32_t* out_lens;
  const float* acc;
  int64_t acc_len;
  int32_t* kept;                    // [B, hkv, budget]
  float* acc_out;
  int64_t acc_out_len;
  int* status;
  int budget, sink, recent;
};

struct CacheAppendLaunch {
  CacheView c;
  DraftView d;                      // tokens, k_new, v_new
  const int32_t* src;
  const int32_t* counts;
  int32_t* lens_out;
  int* status;
};

struct CacheSelectLaunch {
  CacheView c;
  DraftView d;
  int32_t* pages;
  int32_t* sel_table;
  int32_t* sel_lens;
  int* status;
  int n_select, sink, recent;
};

cudaError_t launch_cache_attn(const CacheAttnLaunch& L, cudaStream_t stream);
cudaError_t launch_cache_evidence(const CacheEvidenceLaunch& L, cudaStream_t stream);
cudaError_t launch_cache_evict(const CacheEvictLaunch& L, cudaStream_t stream);
cudaError_t launch_cache_append(const CacheAppendLaunch& L, cudaStream_t stream);
cudaError_t launch_cache_select(const CacheSelectLaunch& L, cudaStream_t stream);

// Row tile and CTAs of a call with `rows` rows of `tokens` drafted tokens for each of `problems` (sequence, KV
// head) pairs, whose tables hold up to `capacity` tokens.
struct CacheAttnShape {
  int tile_rows, row_tiles, slots, slot_rows, key_tile, n_ctas, min_units, lead, join_warps;
  bool wide, join_tile;
};
CacheAttnShape cache_attn_shape(int rows, int tokens, int64_t problems, int64_t capacity, int head_dim, const QueryTile& qt,
                                bool q_map, int n_sm);
cudaError_t launch_cache_attn_wide(const CacheAttnLaunch& L, cudaStream_t stream);

// What the cache calls use of a workspace (evisel_capi.cpp).
struct WsCache {
  void* buf = nullptr;              // scratch of the calls
  size_t bytes = 0;
  std::vector<void*> outgrown;      // earlier ones, whose addresses graphs may hold
  size_t held = 0;                  // bytes of all of them
};
int ws_acquire(evisel_ws** inout);  // creates one where *inout is null
WsCache& ws_cache(evisel_ws* ws);
int* ws_status(evisel_ws* ws);
void ws_ran_on(evisel_ws* ws, cudaStream_t stream);
// 4-D map of `dims` with byte strides `strides` of dims 1..3, 128-byte swizzle; dtype as evisel_cache's.
int encode_map4(CUtensorMap* map, const void* base, int dtype, const uint64_t (&dims)[4], const uint64_t (&strides)[3],
                const uint32_t (&box)[4]);

}  // namespace evisel
