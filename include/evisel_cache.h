/*
 * evisel_cache.h - C ABI of the paged key/value cache that follows the probe.
 *
 * The prefill leaves keys and values; the text rows' attention says which
 * visual tokens matter (Sec. 3.2, "Evidence Decomposition"). These calls keep
 * that cache while the model answers: append tokens, attend from drafted
 * tokens, accumulate attention weight per cached token, cut the cache down to
 * a budget by that weight, and read only the pages a cheap score selects (the
 * block means of Appendix Eq. 7, per query instead of per prefill row). The
 * paper has no counterpart to the calls themselves.
 *
 * The conventions of evisel.h hold: device and host pointers, `stream`, return
 * codes with evisel_last_error(), and a workspace that a call creates when
 * *ws_inout == NULL, which evisel_status() reads and evisel_free() releases.
 * Beyond them:
 *   - Lengths, page tables, tree bits and counts are device memory, read by the
 *     kernels, so that a captured graph replays with new ones. A length outside
 *     [0, max_pages * page], a page id outside [0, n_pages), a source index
 *     outside the new tokens or an append past the table is caught by the
 *     kernels: no access leaves the buffers, nothing is written to a page that
 *     the sequence's table does not hold, the results of that sequence are
 *     unspecified, and evisel_status() answers EVISEL_EBOUNDS.
 *   - A call allocates only where it creates its workspace or an attention needs
 *     more scratch than it holds, which is refused (EVISEL_EINVAL) while `stream`
 *     is being captured: not with the same or smaller sizes again, so capture
 *     after a first call. Scratch that a larger call outgrew stays until
 *     evisel_free(), and with it the graphs that were captured before.
 */
#ifndef EVISEL_CACHE_H
#define EVISEL_CACHE_H

#include "evisel.h"

#ifdef __cplusplus
extern "C" {
#endif

#define EVISEL_BF16 0
#define EVISEL_FP16 1

/* A paged cache. Token i of sequence b is slot i % page of page
 * table[b][i / page]; its key for KV head h is
 *   k + id * k_stride[0] + h * k_stride[1] + slot * k_stride[2]   (elements).
 * A view that has its own pages per KV head (evisel_cache_select) has
 * table_stride[1] and lens_stride[1] != 0. */
typedef struct {
  int32_t batch;               /* sequences, >= 0                                        */
  int32_t hkv;                 /* KV heads                                               */
  int32_t head_dim;            /* d in {64, 128}                                         */
  int32_t page;                /* tokens per page: 16, 32, 64 or 128                     */
  int32_t n_pages;             /* pages of the pool                                      */
  int32_t max_pages;           /* entries of a table row                                 */
  int32_t dtype;               /* EVISEL_BF16 or EVISEL_FP16, of everything but lse, acc */
  int32_t reserved;            /* 0                                                      */
  int64_t k_stride[3];         /* page, head, token, in elements; multiples of 8; d is   */
  int64_t v_stride[3];         /*   contiguous                                           */
  int64_t table_stride[2];     /* sequence, head (0: shared by the heads)                */
  int64_t lens_stride[2];      /* sequence, head (0: shared)                             */
  void* k;                     /* device, 16-byte aligned                                */
  void* v;
  const int32_t* table;        /* device                                                 */
  int32_t* lens;               /* device: tokens cached                                  */
  void* k_mean;                /* device [n_pages, hkv, d] contiguous, 16-byte aligned,
                                  or NULL: mean key of each page's tokens (Eq. 7)        */
} evisel_cache;

/* Drafted tokens: the T = `tokens` new tokens of each sequence, T = 1 in plain
 * decoding. Token t of sequence b attends every cached token of b and those
 * drafted tokens j < drafted[b] whose bit is set: bit j % 32 of
 * tree[b * tree_stride[0] + t * tree_stride[1] + j / 32] (a tree's ancestor
 * bits; its own bit is not implied). tree == NULL: the drafted tokens are a
 * chain, j <= t. k_new == NULL: only the cache is attended. */
typedef struct {
  int32_t tokens;              /* T, 1..1024 (0: nothing to do)                          */
  int32_t hq;                  /* query heads, a multiple of hkv, hq / hkv <= 128        */
  float softmax_scale;         /* 0 => 1 / sqrt(head_dim)                                */
  int32_t reserved;            /* 0                                                      */
  int64_t q_stride[3];         /* sequence, token, head, in elements; multiples of 8     */
  int64_t k_new_stride[3];     /* sequence, token, head                                  */
  int64_t v_new_stride[3];
  int64_t tree_stride[2];      /* sequence (0: one tree for all), token                  */
  const void* q;               /* device [B, T, hq, d], 16-byte aligned                  */
  const void* k_new;           /* device [B, T, hkv, d], 16-byte aligned, or NULL        */
  const void* v_new;
  const int32_t* tree;         /* device, or NULL                                        */
  const int32_t* drafted;      /* device [B] or NULL (T each)                            */
} evisel_draft;

/* Attention of the drafted tokens: s = softmax_scale q . k over the allowed
 * keys, LSE = ln sum exp(s), O = sum exp(s - LSE) v; query head h reads KV head
 * h / (hq / hkv). A row without any allowed key, and every row
 * t >= drafted[b], gets O = 0 and LSE = -inf. Values of keys that a row does
 * not attend never enter it, non-finite ones included.
 * Logits, sums and O are held in 32 bits. Weights are rounded to the cache's
 * type for their product with v (the tensor cores' operand type; against 64 bits
 * O is off by 2.3e-3 in bf16 and 2.1e-4 in fp16, by 1.7e-3 and 2.0e-4 if they were
 * not), those of drafted keys only where many drafted rows are joined by tiles;
 * their sum, and so LSE, is not. In fp16 a weight counts down to 2^-32 of the
 * largest. Which kernels run, and where a sequence's keys are cut, goes by the
 * sizes of the whole call: the same call gives the same bits, the same
 * sequence in another batch may differ in the last ones.
 * The choice between few and many rows goes by what the tables could hold, not by
 * the lengths. Queries repeated by a stride of 0 are attended 16 or 32 rows at a time.
 *   o    device [B, T, hq, d] contiguous, 16-byte aligned (written)
 *   lse  device fp32 [hq, B, T], natural log (written)
 * The workspace keeps the fp32 partial results of ranges of cached keys: for
 * tiles of r = 16, 32, 128 or 256 rows (2 SMs + B * hkv * ceil(T * hq / hkv / r))
 * * r * (d + 2) * 4 bytes; with what it outgrew at most 4.5 times as much.
 * Errors: EVISEL_EINVAL, EVISEL_EUNSUPPORTED, EVISEL_ENOMEM, EVISEL_ECUDA. */
int evisel_cache_attention(const evisel_cache* cache, const evisel_draft* draft, void* o, float* lse, void* stream,
                           evisel_ws** ws_inout);

/* Attention weight per cached token:
 *   acc[b, h, m] (+)= sum_{t used} sum_{heads g of group h} exp(softmax_scale q[b, t, g] . k_m - LSE[g, b, t])
 * for m < the sequence's length (entries past it are left alone). With the LSE
 * of evisel_cache_attention() these are the probabilities of that call; rows
 * with LSE = -inf add nothing. Queries repeated by a stride of 0 take a slow
 * kernel without tensor cores (128 rows of 28 heads over 65,536 keys: 15 ms, not
 * 0.07): copy them where there are many.
 *   draft  tokens, hq, softmax_scale, q and drafted (rows t >= drafted[b] add
 *          nothing); the rest is not read
 *   use    device uint8 [B, T] or NULL: only rows whose byte is not 0 add (the
 *          accepted ones of a drafted tree)
 *   acc    device fp32 [B, hkv, acc_len] contiguous, acc_len >= the longest sequence
 *          (NULL with acc_len = 0)
 *   accumulate  0: overwrite, 1: add
 * Errors: EVISEL_EINVAL, EVISEL_EUNSUPPORTED, EVISEL_ENOMEM, EVISEL_ECUDA; a
 * sequence longer than acc_len shows as EVISEL_EBOUNDS in evisel_status(). */
int evisel_cache_evidence(const evisel_cache* cache, const evisel_draft* draft, const float* lse, const uint8_t* use,
                          float* acc, int64_t acc_len, int accumulate, void* stream, evisel_ws** ws_inout);

/* Cuts every (sequence, KV head) down to `budget` tokens: all of them where
 * there are no more; else the first `sink`, the last `recent` and, of the rest,
 * those with the largest acc (ties: the lower position; NaN counts as lowest),
 * in their order. They are copied to the first slots of out's pages.
 *   acc       device fp32 [B, hkv, acc_len], acc_len >= the longest sequence (NULL
 *             with acc_len = 0)
 *   out       another cache of the same batch, heads, head_dim and dtype, with
 *             room for budget tokens per sequence; its pages must not be among
 *             the cache's. k, v, lens and (if given) k_mean are written; page
 *             size and strides may differ
 *   kept      device int32 [B, hkv, budget]: positions kept, ascending, -1 past them
 *   acc_out   device fp32 [B, hkv, acc_out_len] (written), acc_out_len >= budget:
 *             their acc, 0 past them
 * sink, recent >= 0, sink + recent <= budget, budget >= 1.
 * Errors: EVISEL_EINVAL, EVISEL_EUNSUPPORTED, EVISEL_ENOMEM, EVISEL_ECUDA. */
int evisel_cache_evict(const evisel_cache* cache, const float* acc, int64_t acc_len, const evisel_cache* out,
                       int32_t budget, int32_t sink, int32_t recent, int32_t* kept, float* acc_out,
                       int64_t acc_out_len, void* stream, evisel_ws** ws_inout);

/* Appends tokens: the i-th of sequence b, i < counts[b], is new token src[b, i]
 * and goes to position lens[b] + i. lens_out[b] = lens[b] + counts[b]; lens
 * itself is not written. With k_mean, the means of the touched pages are formed
 * again over all their tokens (fp32 sums in a fixed order, rounded once).
 *   draft   tokens (any number here), k_new and v_new with strides; the rest is not read
 *   src     device int32 [B, T] or NULL (token i itself)
 *   counts  device int32 [B], 0..T, or NULL (T each)
 *   lens_out  device int32 [B], apart from the cache's lens and table, src and counts: other
 *             blocks of the call still read them (over the table it is not refused)
 * table and lens must be shared by the heads. A page may belong to one sequence
 * only where tokens go. Errors: EVISEL_EINVAL, EVISEL_EUNSUPPORTED,
 * EVISEL_ENOMEM, EVISEL_ECUDA. */
int evisel_cache_append(const evisel_cache* cache, const evisel_draft* draft, const int32_t* src,
                        const int32_t* counts, int32_t* lens_out, void* stream, evisel_ws** ws_inout);

/* Chooses pages for every (sequence, KV head): all where there are at most
 * n_select; else the first `sink`, the last `recent` and, of the rest, those
 * with the largest score
 *   score_j = max over t < drafted[b] and the heads of the group of q . k_mean_j,
 * so that all drafted tokens and heads of a group share one choice
 * (fp32; ties: the lower page; a NaN product counts as -inf), in order. The result is a
 * cache view for evisel_cache_attention(): the cache with table = sel_table,
 * table_stride = {hkv * n_select, n_select}, max_pages = n_select, lens =
 * sel_lens, lens_stride = {hkv, 1}; the last page keeps its place, so that only
 * the last may be short.
 *   pages      device int32 [B, hkv, n_select]: chosen logical pages, -1 past them
 *   sel_table  device int32 [B, hkv, n_select]: their page ids, -1 past them
 *   sel_lens   device int32 [B, hkv]: tokens of the chosen pages
 * sink >= 0, recent >= 1, sink + recent <= n_select; max_pages <= 8192.
 * Errors: EVISEL_EINVAL (also: k_mean is NULL), EVISEL_EUNSUPPORTED,
 * EVISEL_ENOMEM, EVISEL_ECUDA. */
int evisel_cache_select(const evisel_cache* cache, const evisel_draft* draft, int32_t n_select, int32_t sink,
                        int32_t recent, int32_t* pages, int32_t* sel_table, int32_t* sel_lens, void* stream,
                        evisel_ws** ws_inout);

#ifdef __cplusplus
}
#endif

#endif /* EVISEL_CACHE_H */
