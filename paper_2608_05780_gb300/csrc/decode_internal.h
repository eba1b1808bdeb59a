// Structures shared by the host side of the decoding-step calls
// (evisel_decode.cpp) and their kernels. Not part of the public ABI.
#pragma once

#include "cache_internal.h"

namespace evisel {

struct RopeView {
  uint64_t turn[64];                // 2^-64 turns per position of pair i
  int pairs;                        // r / 2
  int interleaved;
  int border[2];                    // pairs below border[0] read axis 0, below border[1] axis 1, the others axis 2
  float scale;
};

struct PositionView {
  const int32_t* at;
  const int32_t* first;
  int64_t stride[2];                // axis, sequence
};

struct HeadsView {
  const void* in;
  void* out;
  int64_t is[3], os[3];             // sequence, token, head (elements)
  int heads;
};

struct RotaryLaunch {
  RopeView rope;
  PositionView pos;
  HeadsView q, k;                   // k.heads = 0: none
  int batch, tokens, head_dim, dtype;
  int transpose;
};

struct AppendRotaryLaunch {
  RopeView rope;
  PositionView pos;
  CacheAppendLaunch a;
  HeadsView q;                      // heads = 0: none
};

constexpr int kMaxBeams = 64, kMaxBeamsOut = 64;

struct BeamLaunch {
  const void* logits;
  int64_t ls[2];                    // sequence, beam (elements)
  const float* scores;
  const uint8_t* finished;
  float* score_out;
  int32_t* parent;
  int32_t* token;
  uint8_t* ended_out;
  float2* part;                     // [rows, blocks]: maximum, sum of exponentials
  int batch, beams, vocab, n, dtype, pad, eos;
  int row_vectors, block_vectors, block_shift, ctas, small;   // as BeamSplit's
  unsigned blocks, total;                            // of a row, of all rows
  unsigned step;                                     // warps: step_batch sequences, step_beam beams and step_block blocks
  int step_batch, step_beam, step_block;
  unsigned inverse_blocks;                           // 2^32 / blocks, rounded up: i / blocks = umulhi(i, inverse_blocks)
};

constexpr int kMaxStates = 8;

struct ReorderLaunch {
  CacheView c;
  void* k;
  void* v;
  void* k_mean;
  const int32_t* parent;
  int32_t* table_out;
  int32_t* lens_out;
  int* status;
  int beams, n_states;
  int heads;                        // of a block
  const char* in[kMaxStates];
  char* out[kMaxStates];
  int64_t row_bytes[kMaxStates];
  int first_block[kMaxStates + 1];  // state i's blocks, behind those of the cache
  int chunks[kMaxStates];           // blocks of a row
};

// A row of row_vectors 16-byte vectors as `blocks` blocks of block_vectors, which `warps` warps of `ctas` CTAs take in turn.
struct BeamSplit {
  int row_vectors, block_vectors, block_shift, blocks, ctas, warps;   // block_vectors = 1 << block_shift
  int small;                                         // one launch: the warps are those of a sequence's cluster
};
BeamSplit beam_split(int64_t rows, int beams, int vocab, int n, int dtype, int n_sm);

cudaError_t launch_rotary(const RotaryLaunch& L, cudaStream_t stream);
cudaError_t launch_append_rotary(const AppendRotaryLaunch& L, cudaStream_t stream);
cudaError_t launch_beams(const BeamLaunch& L, cudaStream_t stream);
cudaError_t launch_reorder(const ReorderLaunch& L, cudaStream_t stream);
// Bytes of a state row that a block copies, and of a page's keys and values at most where it takes several heads.
constexpr int kStateBytes = 16384, kPageBytes = 32768;

}  // namespace evisel
