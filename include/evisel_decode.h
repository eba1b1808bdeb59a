/*
 * evisel_decode.h - C ABI of what a decoding step needs around the attention over
 * the paged cache of evisel_cache.h: the position rotation of queries and keys,
 * by itself or on the way into the cache, the selection of beams from the logits,
 * and the reordering of the beams' caches and other states.
 *
 * The paper has no counterpart to these calls. The conventions of evisel.h and
 * evisel_cache.h hold: device memory is checked by the kernels (nothing leaves the
 * buffers, evisel_status() answers EVISEL_EBOUNDS), a call allocates only where it
 * creates its workspace or needs more scratch than it holds.
 */
#ifndef EVISEL_DECODE_H
#define EVISEL_DECODE_H

#include "evisel_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

#define EVISEL_FP32 2              /* logits only */

/* A position rotation of the first r = rotary_dim dimensions of a head, r / 2
 * pairs: pair i is (x[i], x[i + r / 2]), or with `interleaved` (x[2 i], x[2 i + 1]).
 * At position p its angle is a = p f_i:
 *   y1 = scale (x1 cos a - x2 sin a),  y2 = scale (x2 cos a + x1 sin a);
 * dimensions r.. stay. With axes = 3 the first section[0] pairs read the position on
 * axis 0 (time), the next section[1] on axis 1, the last section[2] on axis 2.
 * evisel_rope_init() fills in everything; interleaved, axes, section and scale may
 * be changed after it. */
typedef struct {
  int32_t rotary_dim;              /* r: a multiple of 16, at most head_dim           */
  int32_t interleaved;             /* 0 or 1                                          */
  int32_t axes;                    /* 1 or 3                                          */
  int32_t section[3];              /* with 3 axes: pairs of each, r / 2 together      */
  float scale;                     /* of the rotated dimensions, finite               */
  int32_t reserved;                /* 0                                               */
  uint64_t turn[64];               /* f_i / 2 pi modulo 1, in units of 2^-64 of a turn:
                                      p * turn[i] modulo 2^64 is the angle of any 32-bit
                                      position, off from p f_i / 2 pi (f_i in fp64) by at
                                      most |p| max(1, |f_i| / 2 pi) 2^-52 turns        */
} evisel_rope;

/* Frequencies f_i = base^(-2 i / r), in radians per position; or freq_h[i] (host,
 * r / 2 values, finite) where freq_h is not NULL, base then not read. For contexts longer than the
 * trained one: original = 0 divides every f_i by factor; original > 0 (the trained
 * length) goes by how often a pair turns over it, n_i = original f_i / (2 pi):
 *   f_i (g_i + (1 - g_i) / factor),  g_i = (n_i - low_turns) / (high_turns - low_turns), within 0 and 1,
 * so that fast pairs stay and slow ones are stretched. factor = 1: neither.
 * Errors: EVISEL_EINVAL, EVISEL_EUNSUPPORTED. */
int evisel_rope_init(evisel_rope* rope, int32_t rotary_dim, double base, double factor, double original,
                     double low_turns, double high_turns, const double* freq_h);

/* Where tokens stand: token t of sequence b is at position
 *   at[axis * stride[0] + b * stride[1] + t]    (at != NULL),
 *   first[b] + t                                (on every axis; first != NULL),
 *   t, in an append: the token's place in the cache    (both NULL).
 * Any int32, negative ones too. */
typedef struct {
  const int32_t* at;               /* device or NULL                                  */
  const int32_t* first;            /* device [B] or NULL; not with at                 */
  int64_t stride[2];               /* of at, in elements: axis, sequence; 0 to below 2^38 */
} evisel_positions;

/* Heads [B, T, heads, d] to rotate. */
typedef struct {
  int32_t batch, tokens, heads;    /* >= 0                                            */
  int32_t head_dim;                /* 64 or 128                                       */
  int32_t dtype;                   /* EVISEL_BF16 or EVISEL_FP16                      */
  int32_t reserved;                /* 0                                               */
  int64_t in_stride[3];            /* sequence, token, head, in elements; multiples of 8 */
  int64_t out_stride[3];           /* likewise, and not 0                             */
  const void* in;                  /* device, 16-byte aligned                         */
  void* out;                       /* device; `in` itself with the same strides, or memory
                                      apart from it; apart from the positions         */
} evisel_heads;

/* Rotates q and (unless NULL) k, which have the same batch, tokens, head_dim and
 * dtype, to the positions of their tokens. Products in fp32, rounded once.
 * transpose = 1 applies the transposed matrix (scale included): the gradient of the
 * inputs from that of the outputs, and where scale is 1 the way back. No workspace;
 * nothing is checked on the device. k's memory shares nothing with q's output, nor
 * q's with k's, but for both in place in the rows of one tensor.
 * Errors: EVISEL_EINVAL, EVISEL_EUNSUPPORTED, EVISEL_ECUDA. */
int evisel_rotary(const evisel_rope* rope, const evisel_heads* q, const evisel_heads* k, const evisel_positions* positions,
                  int transpose, void* stream);

/* evisel_cache_append() of keys that are rotated on the way: new token j of sequence
 * b, the i-th to be appended (j = src[b, i], or i), has the position that `positions`
 * names for token j; with `first` or without any it is first[b] + i or lens[b] + i.
 * Keys are rounded once, after the rotation; page means are those of the keys as
 * stored. Values are copied. With draft->q the step's queries [B, T, hq, d] are
 * rotated in the same launch, all T of each sequence, token t as token t (without
 * `at` this needs src == NULL).
 *   draft  tokens, k_new and v_new with strides; hq, q and q_stride, or q == NULL
 *   q_out  device [B, T, hq, d] contiguous, 16-byte aligned (written): q itself where that
 *          is contiguous, or memory apart from every input, lens_out and the cache; NULL without q
 * Everything else as in evisel_cache_append(): src, counts, lens_out (here refused over the
 * table and the positions, too).
 * Errors: EVISEL_EINVAL, EVISEL_EUNSUPPORTED, EVISEL_ENOMEM, EVISEL_ECUDA. */
int evisel_cache_append_rotary(const evisel_cache* cache, const evisel_rope* rope, const evisel_draft* draft,
                               const evisel_positions* positions, const int32_t* src, const int32_t* counts,
                               int32_t* lens_out, void* q_out, void* stream, evisel_ws** ws_inout);

/* One step of a beam search. */
typedef struct {
  int32_t batch;                   /* sequences, >= 0                                 */
  int32_t beams;                   /* K of each, 1..64                                */
  int32_t vocab;                   /* V, 1..2^24                                      */
  int32_t n_out;                   /* n, 1..64                                        */
  int32_t dtype;                   /* of the logits: EVISEL_BF16, _FP16, _FP32        */
  int32_t pad;                     /* token of an ended beam, 0 <= pad < V            */
  int32_t eos;                     /* token that ends a beam; -1: none                */
  int32_t reserved;                /* 0                                               */
  int64_t logits_stride[2];        /* sequence, beam, in elements, 0 to below 2^38    */
  const void* logits;              /* device [B, K, V], V contiguous                  */
  const float* scores;             /* device [B, K]: summed log-probabilities, or NULL: 0 */
  const uint8_t* finished;         /* device [B, K] or NULL: not 0 where a beam has ended */
} evisel_beams;

/* The n highest of all continuations (k, v) of a sequence by
 *   scores[b, k] + x_kv - ln sum_w exp(x_kw),   x = logits[b],
 * in descending order, ties in ascending order of (k, v). A beam that has ended has
 * one continuation, (k, pad) with its score; its logits are not read. A value that is
 * -inf or NaN is none: a forbidden token (-inf), a beam without a score (-inf), all
 * of a row with a NaN or +inf logit, a beam whose score is NaN or +inf.
 * Outputs are apart from the inputs and from one another; B K is at most 65,535.
 *   score_out  device fp32 [B, n] (written), -inf past the continuations there are
 *   parent     device int32 [B, n]: k, -1 past them
 *   token      device int32 [B, n]: v, -1 past them
 *   ended_out  device uint8 [B, n] or NULL: 1 where the parent had ended, where v is
 *              eos, and past them
 * Within a beam the order is that of the logits, exactly, also where a large score leaves less of
 * them in their values; between beams it goes by values of 48
 * bits whose normaliser is formed from fp32 exponentials, fp32 sums of blocks of 1,024 of them (512 of fp32 logits; powers of
 * two more for long rows) and 48-bit sums of those: off by 2^-18 at most, 1e-7 as a rule. Equal rows have the
 * same normaliser wherever they lie, and the same call gives the same bits. Rows that begin on 16 bytes are read fastest.
 * The workspace keeps 8 bytes for every 1,024 logits (512 in fp32).
 * Errors: EVISEL_EINVAL, EVISEL_EUNSUPPORTED, EVISEL_ENOMEM, EVISEL_ECUDA. */
int evisel_beam_select(const evisel_beams* beams, float* score_out, int32_t* parent, int32_t* token, uint8_t* ended_out,
                       void* stream, evisel_ws** ws_inout);

/* One array of states by sequence: row c of `out` becomes the row of c's parent. */
typedef struct {
  const void* in;                  /* device [batch, row_bytes]                       */
  void* out;                       /* device [batch, row_bytes], apart from every input and
                                      (not refused) from the cache's pages and means    */
  int64_t row_bytes;
} evisel_state;

/* The beams that go on. The cache's batch is groups of K = `beams` sequences of one
 * length; sequence j of group g takes over from sequence parent[g, j] of its group (from
 * itself where that is negative: a slot without a continuation). Full pages are shared:
 *   table_out[c, m] = table[p, m] for m < lens[p] / page          (p: c's parent),
 *   table_out[c, m] = table[donor, m] from there on, lens_out[c] = lens[p].
 * The pages from the one in progress on are a sequence's own: the first child of p
 * keeps p's, the e-th of a group's further children takes those of its e-th sequence without
 * a child, and gets the tokens of p's page in progress (keys, values and, with
 * k_mean, its mean) copied into its first. So from the pages in progress on no page is
 * lost or used twice, and none is allocated. Before them the children of a parent share its pages, and full
 * pages of a sequence without a child are in no table any more, unless others share them: a caller that
 * gives pages back counts the tables that name them, and finds those that left as the pages that a
 * group's rows of `table` name and its rows of table_out do not. A sequence without a child may be shorter than the parent whose child
 * takes its pages (the empty slots beside a prompt); longer by whole pages shows as EVISEL_EBOUNDS,
 * as does a parent >= K, which counts as negative, and the group's result is unspecified.
 *   cache      table and lens shared by the heads; batch a multiple of beams
 *   parent     device int32 [batch / beams, beams]
 *   states     host array [n_states] of up to 8 others
 *   table_out  device int32 [batch, max_pages] contiguous, not the cache's own
 *   lens_out   device int32 [batch], not the cache's own
 * Errors: EVISEL_EINVAL, EVISEL_EUNSUPPORTED, EVISEL_ENOMEM, EVISEL_ECUDA. */
int evisel_cache_reorder(const evisel_cache* cache, const int32_t* parent, int32_t beams, const evisel_state* states,
                         int32_t n_states, int32_t* table_out, int32_t* lens_out, void* stream, evisel_ws** ws_inout);

#ifdef __cplusplus
}
#endif

#endif /* EVISEL_DECODE_H */
