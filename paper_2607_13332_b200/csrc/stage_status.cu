// The status word that the library keeps for callers who have none (include/agora_stage.h).
#include <cuda_runtime.h>

#include "agora_stage.h"

namespace {
__device__ int32_t g_status_word;   // 0 when the module is loaded, on every device
}

extern "C" int32_t *stage_status_word(void) {
  // The first call may be within a stream capture: the lookup loads the module, which a capture lets pass in relaxed mode only.
  cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
  const bool relaxed = cudaThreadExchangeStreamCaptureMode(&mode) == cudaSuccess;
  void *at = nullptr;
  if (cudaGetSymbolAddress(&at, g_status_word) != cudaSuccess) {
    cudaGetLastError();
    at = nullptr;
  }
  if (relaxed) cudaThreadExchangeStreamCaptureMode(&mode);
  return static_cast<int32_t *>(at);
}
