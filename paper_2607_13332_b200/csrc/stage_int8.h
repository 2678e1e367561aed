// Host-side entry to the 8-bit product's kernels.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace ssn {

struct Int8Matmul {
  const int8_t *xq, *wq;
  const float *xs, *ws;
  void *y;
  int64_t ldx, ldw, ldy, n, inner, outer;
  int32_t *dev_status;
};

// tcgen05 kernels: operand rows on 16-byte boundaries.  cudaErrorNotSupported, with nothing launched, for others.
cudaError_t launch_int8_umma(const Int8Matmul &a, bool f32, int sm_count, cudaStream_t stream);

}  // namespace ssn
