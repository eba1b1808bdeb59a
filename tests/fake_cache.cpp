// The cache kernels' launchers for fake_cuda.cpp's stand-in runtime: each counts
// its launches and can be made to fail once.
#include <cuda_runtime.h>

#include "cache_internal.h"

extern "C" {

static int g_launches = 0, g_fail = 0;
void fake_fail_launch(int n) { g_fail = n; }
int fake_launches() { return g_launches; }

}  // extern "C"

namespace evisel {

static cudaError_t launched() {
  ++g_launches;
  return g_fail > 0 && --g_fail == 0 ? cudaErrorLaunchOutOfResources : cudaSuccess;
}
cudaError_t launch_cache_attn(const CacheAttnLaunch&, cudaStream_t) { return launched(); }
cudaError_t launch_cache_evidence(const CacheEvidenceLaunch&, cudaStream_t) { return launched(); }
cudaError_t launch_cache_evict(const CacheEvictLaunch&, cudaStream_t) { return launched(); }
cudaError_t launch_cache_append(const CacheAppendLaunch&, cudaStream_t) { return launched(); }
cudaError_t launch_cache_select(const CacheSelectLaunch&, cudaStream_t) { return launched(); }
CacheAttnShape cache_attn_shape(int rows, int, int64_t, int64_t, int, const QueryTile&, bool, int n_sm) {
  CacheAttnShape s{};
  s.tile_rows = s.slot_rows = 32;
  s.row_tiles = (rows + 31) / 32;
  s.slots = 1;
  s.key_tile = 64;
  s.n_ctas = 2 * n_sm;
  s.min_units = 1;
  return s;
}

}  // namespace evisel

// A stream capture for the stand-in runtime.
static int g_capturing = 0;
extern "C" void fake_capture(int on) { g_capturing = on; }
extern "C" cudaError_t cudaStreamIsCapturing(cudaStream_t, cudaStreamCaptureStatus* s) {
  return *s = g_capturing ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone, cudaSuccess;
}
