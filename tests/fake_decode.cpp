// The decoding-step kernels' launchers for fake_cuda.cpp's stand-in runtime: the
// last launch is kept for the tests to look at.
#include <cuda_runtime.h>

#include "decode_internal.h"

static int g_launches = 0, g_fail = 0;
static evisel::RotaryLaunch g_rotary;
static evisel::ReorderLaunch g_reorder;

static cudaError_t launched() {
  ++g_launches;
  return g_fail > 0 && --g_fail == 0 ? cudaErrorLaunchOutOfResources : cudaSuccess;
}

namespace evisel {
cudaError_t launch_rotary(const RotaryLaunch& L, cudaStream_t) { return g_rotary = L, launched(); }
cudaError_t launch_append_rotary(const AppendRotaryLaunch&, cudaStream_t) { return launched(); }
cudaError_t launch_beams(const BeamLaunch&, cudaStream_t) { return launched(); }
cudaError_t launch_reorder(const ReorderLaunch& L, cudaStream_t) { return g_reorder = L, launched(); }
BeamSplit beam_split(int64_t, int, int vocab, int, int, int) { return {vocab / 8 + 1, 128, 7, vocab / 1024 + 1, 304, 4864, 0}; }
}  // namespace evisel

extern "C" {
void fake_fail_decode(int n) { g_fail = n; }
int fake_decode_launches() { return g_launches; }
int fake_axis_of_pair(int i) { return i < g_rotary.rope.border[0] ? 0 : i < g_rotary.rope.border[1] ? 1 : 2; }
int fake_reorder_blocks(int i) { return g_reorder.first_block[i]; }
}
