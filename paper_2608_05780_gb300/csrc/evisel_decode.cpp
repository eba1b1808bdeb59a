// Host side of the decoding-step calls (evisel_decode.h): argument checks,
// scratch of the workspace and kernel launches.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <string>

#include <cuda_runtime.h>

#include "../../include/evisel_decode.h"
#include "cache_host.h"
#include "decode_internal.h"

using namespace evisel;
using namespace evisel::host;

namespace {

constexpr int kMaxPairs = 64;
constexpr int64_t kMaxTokens = int64_t(1) << 30;
constexpr int64_t kMaxRows = 65535;              // of logits, as many as a cache has sequences
constexpr int kMaxVocab = 1 << 24;

Strided heads_of(const void* p, const int64_t* stride, const int64_t* sizes, int head_dim) {
  return {p, 2, head_dim, 3, {sizes[0], sizes[1], sizes[2]}, {stride[0], stride[1], stride[2]}};
}

// Heads [batch, token, head, d] in memory.
struct HeadsAt {
  const void* p;
  const int64_t* stride;
  int64_t heads;
};

// Whether two of them, of the same batch and tokens, share no memory: apart as wholes, or parts of the rows of
// one tensor, where dimensions of one stride step over both.
bool apart(const HeadsAt& a, const HeadsAt& b, int64_t batch, int64_t tokens, int head_dim) {
  using Wide = __int128;
  const Wide from = static_cast<Wide>(reinterpret_cast<uintptr_t>(b.p)) - reinterpret_cast<uintptr_t>(a.p);
  const int64_t sizes[2] = {batch, tokens};
  const auto step = [&](const HeadsAt& h, int i) { return 2 * (sizes[i] > 1 ? static_cast<Wide>(h.stride[i]) : 0); };
  for (int rows = 0; rows < 4; ++rows) {         // the dimensions that step over both: bit 0 the batch's, bit 1 the tokens'
    const auto reach = [&](const HeadsAt& h) {
      Wide bytes = 2 * (head_dim + (h.heads > 1 ? (h.heads - 1) * static_cast<Wide>(h.stride[2]) : 0));
      for (int i = 0; i < 2; ++i) bytes += rows >> i & 1 ? 0 : (sizes[i] - 1) * step(h, i);
      return bytes;
    };
    const Wide ends[2] = {reach(a), from + reach(b)};
    if (from < ends[0] && 0 < ends[1]) continue;
    Wide both = std::max(ends[0], ends[1]) - std::min<Wide>(0, from);
    bool nested = true;
    const int inner = step(a, 0) < step(a, 1) ? 0 : 1;
    for (const int i : {inner, 1 - inner}) {
      if (!(rows >> i & 1) || sizes[i] <= 1) continue;
      nested = nested && step(a, i) == step(b, i) && both <= step(a, i);
      both += (sizes[i] - 1) * step(a, i);
    }
    if (nested) return true;
  }
  return false;
}

int check_rope(const evisel_rope* r, int head_dim) {
  if (!r) return fail(EVISEL_EINVAL, "rope is NULL");
  if (r->rotary_dim < 16 || r->rotary_dim % 16 != 0 || r->rotary_dim > head_dim)
    return fail(EVISEL_EUNSUPPORTED, "rotary_dim must be a multiple of 16 up to head_dim, got " + std::to_string(r->rotary_dim));
  if (r->interleaved != 0 && r->interleaved != 1) return fail(EVISEL_EINVAL, "interleaved must be 0 or 1");
  if (r->axes != 1 && r->axes != 3) return fail(EVISEL_EUNSUPPORTED, "axes must be 1 or 3");
  if (r->axes == 3) {
    const int32_t* s = r->section;
    if (s[0] < 0 || s[1] < 0 || s[2] < 0 || static_cast<int64_t>(s[0]) + s[1] + s[2] != r->rotary_dim / 2)
      return fail(EVISEL_EINVAL, "sections must not be negative, and rotary_dim / 2 together");
  }
  if (!std::isfinite(r->scale)) return fail(EVISEL_EINVAL, "scale must be finite");
  if (r->reserved != 0) return fail(EVISEL_EINVAL, "reserved must be 0");
  return EVISEL_OK;
}

RopeView view_of(const evisel_rope* r) {
  RopeView v{};
  v.pairs = r->rotary_dim / 2;
  std::copy(r->turn, r->turn + v.pairs, v.turn);
  v.interleaved = r->interleaved;
  v.border[0] = r->axes == 3 ? r->section[0] : v.pairs;
  v.border[1] = r->axes == 3 ? r->section[0] + r->section[1] : v.pairs;
  v.scale = r->scale;
  return v;
}

int check_positions(const evisel_positions* p) {
  if (!p) return fail(EVISEL_EINVAL, "positions is NULL");
  if (p->at && p->first) return fail(EVISEL_EINVAL, "positions: at or first, not both");
  if (misaligned(p->at, 4) || misaligned(p->first, 4)) return fail(EVISEL_EINVAL, "positions must be 4-byte aligned");
  if (p->at && (std::min(p->stride[0], p->stride[1]) < 0 || std::max(p->stride[0], p->stride[1]) >= kMaxStride))
    return fail(EVISEL_EINVAL, "position strides must be 0 to below 2^38");
  return EVISEL_OK;
}

// Whether the bytes hold any of the positions that a call reads.
bool meets_positions(const Range& out, const evisel_positions* p, int axes, int64_t batch, int64_t tokens) {
  return meets(out, {p->at, 4, tokens, 2, {axes, batch}, {p->stride[0], p->stride[1]}}) || out.meets(range_of(p->first, 4 * batch));
}

PositionView view_of(const evisel_positions* p) {
  PositionView v{};
  v.at = p->at;
  v.first = p->first;
  std::copy(p->stride, p->stride + 2, v.stride);
  return v;
}

int check_heads(const evisel_heads* h, const char* what) {
  if (!h) return fail(EVISEL_EINVAL, std::string(what) + " is NULL");
  if (h->head_dim != 64 && h->head_dim != 128)
    return fail(EVISEL_EUNSUPPORTED, "head_dim must be 64 or 128, got " + std::to_string(h->head_dim));
  if (h->dtype != EVISEL_BF16 && h->dtype != EVISEL_FP16) return fail(EVISEL_EUNSUPPORTED, "dtype must be bf16 or fp16");
  if (h->batch < 0 || h->tokens < 0 || h->heads < 0) return fail(EVISEL_EINVAL, "a size is negative");
  if (h->reserved != 0) return fail(EVISEL_EINVAL, "reserved must be 0");
  if (static_cast<int64_t>(h->batch) * h->tokens > kMaxTokens || h->heads > 65535)
    return fail(EVISEL_EUNSUPPORTED, "batch * tokens must be at most 2^30, heads 65535");
  if (h->batch == 0 || h->tokens == 0 || h->heads == 0) return EVISEL_OK;
  if (!h->in || !h->out) return fail(EVISEL_EINVAL, std::string(what) + ": in or out is NULL");
  if (misaligned(h->in) || misaligned(h->out)) return fail(EVISEL_EINVAL, std::string(what) + " must be 16-byte aligned");
  const int64_t sizes[3] = {h->batch, h->tokens, h->heads};
  int rc = check_strides(h->in_stride, sizes, 3, what);
  if (rc == EVISEL_OK) rc = check_strides(h->out_stride, sizes, 3, what);
  if (rc != EVISEL_OK) return rc;
  bool same = h->in == h->out;
  for (int i = 0; i < 3; ++i) {
    if (sizes[i] > 1 && h->out_stride[i] < h->head_dim)
      return fail(EVISEL_EINVAL, std::string(what) + ": strides of the output must be at least head_dim");
    same = same && (sizes[i] <= 1 || h->in_stride[i] == h->out_stride[i]);
  }
  if (!same && !apart({h->in, h->in_stride, h->heads}, {h->out, h->out_stride, h->heads}, h->batch, h->tokens, h->head_dim))
    return fail(EVISEL_EINVAL, std::string(what) + ": out must be in itself with the same strides, or apart from it");
  return EVISEL_OK;
}

HeadsView view_of(const evisel_heads* h) {
  HeadsView v{};
  v.in = h->in;
  v.out = h->out;
  std::copy(h->in_stride, h->in_stride + 3, v.is);
  std::copy(h->out_stride, h->out_stride + 3, v.os);
  v.heads = h->heads;
  return v;
}

// Rotated heads over positions that other blocks still read. (Runs one by one where all that positions reach is
// met: sequences' rows may hold their heads and, apart from them, their position.)
int check_positions_apart(const evisel_heads* h, const evisel_positions* p, int axes) {
  constexpr int64_t kRuns = 1 << 16, kFar = int64_t(1) << 61;
  if (h->heads == 0) return EVISEL_OK;
  const int64_t sizes[3] = {h->batch, h->tokens, h->heads};
  const Strided out = heads_of(h->out, h->out_stride, sizes, h->head_dim);
  bool met = meets(range_of(p->first, 4 * static_cast<int64_t>(h->batch)), out);
  if (p->at) {
    const __int128 reach = static_cast<__int128>(p->stride[0]) * (axes - 1) + static_cast<__int128>(p->stride[1]) * (h->batch - 1) + h->tokens;
    met = meets(range_of(p->at, static_cast<int64_t>(std::min<__int128>(4 * reach, kFar))), out);
    if (met && static_cast<int64_t>(axes) * h->batch <= kRuns) {
      met = false;
      for (int64_t i = 0; i < static_cast<int64_t>(axes) * h->batch && !met; ++i)
        met = meets(range_of(p->at + i / h->batch * p->stride[0] + i % h->batch * p->stride[1], 4 * static_cast<int64_t>(h->tokens)), out);
    }
  }
  return met ? fail(EVISEL_EINVAL, "an output lies over the positions") : EVISEL_OK;
}

// One input's output over another input (each in its own place is the caller's to answer for: rows of one tensor).
int check_apart(const evisel_heads* a, const evisel_heads* b) {
  if (a->heads == 0 || b->heads == 0) return EVISEL_OK;
  const HeadsAt out = {a->out, a->out_stride, a->heads};
  if (a->out != a->in && !apart(out, {b->in, b->in_stride, b->heads}, a->batch, a->tokens, a->head_dim))
    return fail(EVISEL_EINVAL, "an output lies over the other input");
  if (a->out == b->out || (a->out != a->in && !apart(out, {b->out, b->out_stride, b->heads}, a->batch, a->tokens, a->head_dim)))
    return fail(EVISEL_EINVAL, "the outputs lie over one another");
  return EVISEL_OK;
}

}  // namespace

extern "C" {

int evisel_rope_init(evisel_rope* rope, int32_t rotary_dim, double base, double factor, double original, double low_turns,
                     double high_turns, const double* freq_h) {
  return guarded("evisel_rope_init", [&]() -> int {
    constexpr double kTwoPi = 6.283185307179586476925286766559;
    if (!rope) return fail(EVISEL_EINVAL, "rope is NULL");
    if (rotary_dim < 16 || rotary_dim % 16 != 0 || rotary_dim > 2 * kMaxPairs)
      return fail(EVISEL_EUNSUPPORTED, "rotary_dim must be a multiple of 16 up to 128, got " + std::to_string(rotary_dim));
    if (!freq_h && !(base > 0.0 && std::isfinite(base))) return fail(EVISEL_EINVAL, "base must be positive and finite");
    if (!(factor > 0.0 && std::isfinite(factor)) || !(original >= 0.0 && std::isfinite(original)))
      return fail(EVISEL_EINVAL, "factor must be positive, original not negative, both finite");
    if (original > 0.0 && !(std::isfinite(low_turns) && std::isfinite(high_turns) && low_turns < high_turns))
      return fail(EVISEL_EINVAL, "low_turns must be below high_turns, both finite");
    evisel_rope r{};
    r.rotary_dim = rotary_dim;
    r.axes = 1;
    r.scale = 1.f;
    for (int i = 0; i < rotary_dim / 2; ++i) {
      double f = freq_h ? freq_h[i] : std::pow(base, -2.0 * i / rotary_dim);
      if (original > 0.0) {
        const double turns = original * f / kTwoPi;
        const double keep = std::min(1.0, std::max(0.0, (turns - low_turns) / (high_turns - low_turns)));
        f *= keep + (1.0 - keep) / factor;
      } else {
        f /= factor;
      }
      if (!std::isfinite(f)) return fail(EVISEL_EINVAL, "a frequency is not finite");
      const double turn = f / kTwoPi, part = turn - std::floor(turn);
      r.turn[i] = part < 1.0 ? static_cast<uint64_t>(std::ldexp(part, 64)) : 0;
    }
    *rope = r;
    return EVISEL_OK;
  });
}

int evisel_rotary(const evisel_rope* rope, const evisel_heads* q, const evisel_heads* k, const evisel_positions* positions,
                  int transpose, void* stream) {
  return guarded("evisel_rotary", [&]() -> int {
    int rc = check_heads(q, "q");
    if (rc == EVISEL_OK && k) rc = check_heads(k, "k");
    if (rc == EVISEL_OK) rc = check_rope(rope, q->head_dim);
    if (rc == EVISEL_OK) rc = check_positions(positions);
    if (rc != EVISEL_OK) return rc;
    if (k && (k->batch != q->batch || k->tokens != q->tokens || k->head_dim != q->head_dim || k->dtype != q->dtype))
      return fail(EVISEL_EINVAL, "q and k must have the same batch, tokens, head_dim and dtype");
    if (q->batch == 0 || q->tokens == 0 || q->heads + (k ? k->heads : 0) == 0) return EVISEL_OK;
    if (k) rc = check_apart(q, k);
    if (k && rc == EVISEL_OK) rc = check_apart(k, q);
    if (rc == EVISEL_OK) rc = check_positions_apart(q, positions, rope->axes);
    if (k && rc == EVISEL_OK) rc = check_positions_apart(k, positions, rope->axes);
    if (rc != EVISEL_OK) return rc;
    if (sm_count() <= 0) return fail(EVISEL_ECUDA, "the device's multiprocessors cannot be counted");
    RotaryLaunch L{};
    L.rope = view_of(rope);
    L.pos = view_of(positions);
    L.q = view_of(q);
    if (k) L.k = view_of(k);
    L.batch = q->batch;
    L.tokens = q->tokens;
    L.head_dim = q->head_dim;
    L.dtype = q->dtype;
    L.transpose = transpose != 0;
    const cudaError_t e = launch_rotary(L, static_cast<cudaStream_t>(stream));
    return e != cudaSuccess ? cuda_fail(e, "rotary launch") : EVISEL_OK;
  });
}

int evisel_cache_append_rotary(const evisel_cache* cache, const evisel_rope* rope, const evisel_draft* draft,
                               const evisel_positions* positions, const int32_t* src, const int32_t* counts,
                               int32_t* lens_out, void* q_out, void* stream_ptr, evisel_ws** ws_inout) {
  return guarded("evisel_cache_append_rotary", [&]() -> int {
    int rc = check_append(cache, draft, src, counts, lens_out, ws_inout);
    if (rc == EVISEL_OK) rc = check_rope(rope, cache->head_dim);
    if (rc == EVISEL_OK) rc = check_positions(positions);
    if (rc != EVISEL_OK) return rc;
    if (cache->batch == 0) return EVISEL_OK;
    if (meets(range_of(lens_out, 4 * static_cast<int64_t>(cache->batch)), table_of(cache)))
      return fail(EVISEL_EINVAL, "lens_out must not overlap the cache's table");
    if (overlap(lens_out, cache->batch, positions->first, cache->batch))
      return fail(EVISEL_EINVAL, "lens_out must not overlap the positions");
    if (positions->at && draft->tokens > 0) {
      const int64_t span = positions->stride[0] * (rope->axes - 1) + positions->stride[1] * (cache->batch - 1) + draft->tokens;
      if (overlap(lens_out, cache->batch, positions->at, span)) return fail(EVISEL_EINVAL, "lens_out must not overlap the positions");
    }
    AppendRotaryLaunch L{};
    if (draft->q) {
      if (src && !positions->at) return fail(EVISEL_EINVAL, "q beside src needs positions of its own (at)");
      const evisel_heads h = {cache->batch, draft->tokens, draft->hq, cache->head_dim, cache->dtype, 0,
                              {draft->q_stride[0], draft->q_stride[1], draft->q_stride[2]},
                              {static_cast<int64_t>(draft->tokens) * draft->hq * cache->head_dim,
                               static_cast<int64_t>(draft->hq) * cache->head_dim, cache->head_dim},
                              draft->q, q_out};
      if (draft->hq < 1) return fail(EVISEL_EINVAL, "hq must be positive");
      rc = check_heads(&h, "q");
      if (rc != EVISEL_OK) return rc;
      if (draft->tokens > 0) {
        const int64_t sizes[3] = {cache->batch, draft->tokens, cache->hkv}, rows = static_cast<int64_t>(cache->batch) * draft->tokens;
        const Range out = range_of(q_out, 2 * h.out_stride[0] * cache->batch);
        if (meets(out, heads_of(draft->k_new, draft->k_new_stride, sizes, cache->head_dim)) ||
            meets(out, heads_of(draft->v_new, draft->v_new_stride, sizes, cache->head_dim)))
          return fail(EVISEL_EINVAL, "q_out lies over k_new or v_new");
        // (In its own place it lies where q was: the caller's to answer for.)
        if (q_out != draft->q) {
          if (meets(out, lens_of(cache)) || meets(out, table_of(cache)) || out.meets(range_of(src, 4 * rows)) ||
              out.meets(range_of(counts, 4 * static_cast<int64_t>(cache->batch))) || meets_positions(out, positions, rope->axes, cache->batch, draft->tokens))
            return fail(EVISEL_EINVAL, "q_out lies over lens, the table, src, counts or the positions");
          if (out.meets(range_of(lens_out, 4 * static_cast<int64_t>(cache->batch))) || meets(out, pages_of(cache, cache->k, cache->k_stride)) ||
              meets(out, pages_of(cache, cache->v, cache->v_stride)) ||
              out.meets(range_of(cache->k_mean, 2 * static_cast<int64_t>(cache->n_pages) * cache->hkv * cache->head_dim)))
            return fail(EVISEL_EINVAL, "q_out lies over lens_out or the cache's pages or means");
        }
        L.q = view_of(&h);
      }
    }
    const int n_sm = sm_count();
    if (n_sm <= 0) return fail(EVISEL_ECUDA, "the device's multiprocessors cannot be counted");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    rc = acquire(ws_inout, stream);
    if (rc != EVISEL_OK) return rc;
    L.rope = view_of(rope);
    L.pos = view_of(positions);
    L.a = append_of(cache, draft, src, counts, lens_out, *ws_inout);
    const cudaError_t e = launch_append_rotary(L, stream);
    if (e != cudaSuccess) return cuda_fail(e, "rotated append launch");
    ws_ran_on(*ws_inout, stream);
    return EVISEL_OK;
  });
}

int evisel_beam_select(const evisel_beams* beams, float* score_out, int32_t* parent, int32_t* token, uint8_t* ended_out,
                       void* stream_ptr, evisel_ws** ws_inout) {
  return guarded("evisel_beam_select", [&]() -> int {
    if (!beams) return fail(EVISEL_EINVAL, "beams is NULL");
    if (!ws_inout) return fail(EVISEL_EINVAL, "ws_inout is NULL");
    const evisel_beams& m = *beams;
    if (m.dtype != EVISEL_BF16 && m.dtype != EVISEL_FP16 && m.dtype != EVISEL_FP32)
      return fail(EVISEL_EUNSUPPORTED, "dtype must be bf16, fp16 or fp32");
    if (m.batch < 0) return fail(EVISEL_EINVAL, "batch is negative");
    if (m.beams < 1 || m.beams > kMaxBeams) return fail(EVISEL_EUNSUPPORTED, "beams must be 1 to " + std::to_string(kMaxBeams));
    if (m.n_out < 1 || m.n_out > kMaxBeamsOut) return fail(EVISEL_EUNSUPPORTED, "n_out must be 1 to " + std::to_string(kMaxBeamsOut));
    if (m.vocab < 1 || m.vocab > kMaxVocab) return fail(EVISEL_EUNSUPPORTED, "vocab must be 1 to 2^24");
    if (m.pad < 0 || m.pad >= m.vocab) return fail(EVISEL_EINVAL, "pad must be a token");
    if (m.reserved != 0) return fail(EVISEL_EINVAL, "reserved must be 0");
    const int64_t rows = static_cast<int64_t>(m.batch) * m.beams;
    if (rows > kMaxRows) return fail(EVISEL_EUNSUPPORTED, "batch * beams must be at most 65535");
    if (m.batch == 0) return EVISEL_OK;
    const int size = m.dtype == EVISEL_FP32 ? 4 : 2;
    if (!m.logits || !score_out || !parent || !token) return fail(EVISEL_EINVAL, "logits or an output is NULL");
    if (misaligned(m.logits, size) || misaligned(m.scores, 4) || misaligned(score_out, 4) || misaligned(parent, 4) || misaligned(token, 4))
      return fail(EVISEL_EINVAL, "logits, scores and outputs must be aligned to their elements");
    if (m.logits_stride[0] < 0 || m.logits_stride[1] < 0 || std::max(m.logits_stride[0], m.logits_stride[1]) >= kMaxStride)
      return fail(EVISEL_EINVAL, "logits strides must be 0 to below 2^38");
    const int64_t n = static_cast<int64_t>(m.batch) * m.n_out;
    // Other sequences' blocks still read the inputs, the chosen blocks of the logits again.
    const int64_t reach = (m.batch - 1) * m.logits_stride[0] + (m.beams - 1) * m.logits_stride[1] + m.vocab;
    const Range in[3] = {range_of(m.logits, reach * size), range_of(m.scores, 4 * rows), range_of(m.finished, rows)};
    const Range out[4] = {range_of(score_out, 4 * n), range_of(parent, 4 * n), range_of(token, 4 * n), range_of(ended_out, n)};
    for (int i = 0; i < 4; ++i) {
      for (const Range& r : in)
        if (out[i].meets(r)) return fail(EVISEL_EINVAL, "an output lies over logits, scores or finished");
      for (int j = 0; j < i; ++j)
        if (out[i].meets(out[j])) return fail(EVISEL_EINVAL, "outputs lie over one another");
    }
    const int n_sm = sm_count();
    if (n_sm <= 0) return fail(EVISEL_ECUDA, "the device's multiprocessors cannot be counted");
    const BeamSplit split = beam_split(rows, m.beams, m.vocab, m.n_out, m.dtype, n_sm);
    if (rows > 0x7fffffff / split.blocks) return fail(EVISEL_EUNSUPPORTED, "batch * beams * vocab is beyond the blocks that are counted in 31 bits");
    const size_t parts = static_cast<size_t>(rows) * split.blocks;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    int rc = acquire(ws_inout, stream);
    if (rc == EVISEL_OK) rc = grow(*ws_inout, parts * sizeof(float2), stream);
    if (rc != EVISEL_OK) return rc;
    BeamLaunch L{};
    L.logits = m.logits;
    L.ls[0] = m.logits_stride[0];
    L.ls[1] = m.logits_stride[1];
    L.scores = m.scores;
    L.finished = m.finished;
    L.score_out = score_out;
    L.parent = parent;
    L.token = token;
    L.ended_out = ended_out;
    L.part = static_cast<float2*>(ws_cache(*ws_inout).buf);
    L.batch = m.batch;
    L.beams = m.beams;
    L.vocab = m.vocab;
    L.n = m.n_out;
    L.dtype = m.dtype;
    L.pad = m.pad;
    L.eos = m.eos;
    L.row_vectors = split.row_vectors;
    L.block_vectors = split.block_vectors;
    L.block_shift = split.block_shift;
    L.ctas = split.ctas;
    L.small = split.small;
    L.blocks = split.blocks;
    L.step = split.warps;
    L.step_block = split.warps % split.blocks;
    L.step_beam = split.warps / split.blocks % m.beams;
    L.step_batch = split.warps / split.blocks / m.beams;
    L.total = static_cast<unsigned>(parts);
    L.inverse_blocks = static_cast<unsigned>(((uint64_t(1) << 32) + split.blocks - 1) / split.blocks);
    const cudaError_t e = launch_beams(L, stream);
    if (e != cudaSuccess) return cuda_fail(e, "beam selection launch");
    ws_ran_on(*ws_inout, stream);
    return EVISEL_OK;
  });
}

int evisel_cache_reorder(const evisel_cache* cache, const int32_t* parent, int32_t beams, const evisel_state* states,
                         int32_t n_states, int32_t* table_out, int32_t* lens_out, void* stream_ptr, evisel_ws** ws_inout) {
  return guarded("evisel_cache_reorder", [&]() -> int {
    int rc = check_cache(cache, "cache");
    if (rc != EVISEL_OK) return rc;
    if (!ws_inout) return fail(EVISEL_EINVAL, "ws_inout is NULL");
    if (beams < 1 || beams > kMaxBeams) return fail(EVISEL_EUNSUPPORTED, "beams must be 1 to " + std::to_string(kMaxBeams));
    if (cache->batch % beams != 0) return fail(EVISEL_EINVAL, "the cache's batch must be a multiple of beams");
    if (n_states < 0 || n_states > kMaxStates) return fail(EVISEL_EUNSUPPORTED, "at most " + std::to_string(kMaxStates) + " states");
    if (n_states > 0 && !states) return fail(EVISEL_EINVAL, "states is NULL");
    if (cache->hkv > 1 && (cache->table_stride[1] != 0 || cache->lens_stride[1] != 0))
      return fail(EVISEL_EUNSUPPORTED, "a reordering needs a table and lengths that the heads share");
    if (cache->batch == 0) return EVISEL_OK;
    if (!parent || !lens_out || (cache->max_pages > 0 && !table_out)) return fail(EVISEL_EINVAL, "parent, table_out or lens_out is NULL");
    if (misaligned(parent, 4) || misaligned(table_out, 4) || misaligned(lens_out, 4))
      return fail(EVISEL_EINVAL, "parent, table_out and lens_out must be 4-byte aligned");
    const int64_t batch = cache->batch, entries = batch * cache->max_pages;
    const Range in[3] = {range_of(parent, 4 * batch),
                         range_of(cache->table, cache->max_pages > 0 ? 4 * ((batch - 1) * cache->table_stride[0] + cache->max_pages) : 0),
                         range_of(cache->lens, 4 * ((batch - 1) * cache->lens_stride[0] + 1))};
    Range out[kMaxStates + 2] = {range_of(table_out, 4 * entries), range_of(lens_out, 4 * batch)};
    ReorderLaunch L{};
    L.heads = std::min(cache->hkv, std::max(1, kPageBytes / (cache->page * cache->head_dim * 4)));
    L.first_block[0] = static_cast<int>(batch * ((cache->hkv + L.heads - 1) / L.heads));
    int64_t blocks = L.first_block[0];
    for (int i = 0; i < n_states; ++i) {
      const evisel_state& s = states[i];
      if (s.row_bytes < 0 || s.row_bytes >= (int64_t(1) << 40)) return fail(EVISEL_EINVAL, "row_bytes must be 0 to below 2^40");
      if (s.row_bytes > 0 && (!s.in || !s.out)) return fail(EVISEL_EINVAL, "a state is NULL");
      out[i + 2] = range_of(s.out, s.row_bytes * batch);
      L.in[i] = static_cast<const char*>(s.in);
      L.out[i] = static_cast<char*>(s.out);
      L.row_bytes[i] = s.row_bytes;
      const int64_t chunks = (s.row_bytes + kStateBytes - 1) / kStateBytes;
      blocks += chunks * batch;
      if (blocks > 0x7fffffff) return fail(EVISEL_EUNSUPPORTED, "the states are too large for one call");
      L.chunks[i] = static_cast<int>(chunks);
      L.first_block[i + 1] = static_cast<int>(blocks);
    }
    for (int i = 0; i < n_states + 2; ++i) {
      for (const Range& r : in)
        if (out[i].meets(r)) return fail(EVISEL_EINVAL, "an output lies over parent, the table or the lengths");
      for (int j = 0; j < n_states; ++j)
        if (out[i].meets(range_of(states[j].in, states[j].row_bytes * batch))) return fail(EVISEL_EINVAL, "an output lies over a state");
      for (int j = 0; j < i; ++j)
        if (out[i].meets(out[j])) return fail(EVISEL_EINVAL, "outputs lie over one another");
    }
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    rc = acquire(ws_inout, stream);
    if (rc != EVISEL_OK) return rc;
    L.c = view_of(cache);
    L.k = cache->k;
    L.v = cache->v;
    L.k_mean = cache->k_mean;
    L.parent = parent;
    L.table_out = table_out;
    L.lens_out = lens_out;
    L.status = ws_status(*ws_inout);
    L.beams = beams;
    L.n_states = n_states;
    const cudaError_t e = launch_reorder(L, stream);
    if (e != cudaSuccess) return cuda_fail(e, "reordering launch");
    ws_ran_on(*ws_inout, stream);
    return EVISEL_OK;
  });
}

}  // extern "C"
