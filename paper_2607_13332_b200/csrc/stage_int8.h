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

// tcgen05 kernels.  rows16: all operand rows start on 16-byte boundaries.
cudaError_t launch_int8_umma(const Int8Matmul &a, bool f32, bool rows16, int sm_count, cudaStream_t stream);

#ifdef __CUDACC__
// The first `bytes` (0 .. 16) bytes of v, zeros behind them
__device__ __forceinline__ uint4 first_bytes(uint4 v, int bytes) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int keep = min(max(bytes - 4 * i, 0), 4);
    w[i] = keep == 0 ? 0u : w[i] & (0xffffffffu >> (32 - 8 * keep));
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Bytes [at, at + 16) of a row of `bytes` bytes that starts anywhere, zeros past its end: the one or two aligned 16-byte pieces
// that hold some of them (a piece with a byte of the row in it is memory of the row's buffer), shifted together.  The loads are
// apart from the shifting and without a branch, so that many can be on their way at once; at >= bytes loads the row's first
// bytes, of which row16 then keeps none.
struct Row16 {
  uint4 lo, hi;
};
__device__ __forceinline__ Row16 fetch_row16(const int8_t *row, int at, int bytes) {
  if (at >= bytes) at = 0;
  const uintptr_t p = reinterpret_cast<uintptr_t>(row + at);
  const int off = (int)(p & 15);
  const uint4 *from = reinterpret_cast<const uint4 *>(p - off);
  return {__ldg(from), __ldg(from + (off + min(bytes - at, 16) > 16 ? 1 : 0))};
}
__device__ __forceinline__ uint4 row16(const Row16 &r, const int8_t *row, int at, int bytes) {
  const int off = (int)(reinterpret_cast<uintptr_t>(row + at) & 15), there = min(max(bytes - at, 0), 16);
  const uint32_t w[8] = {r.lo.x, r.lo.y, r.lo.z, r.lo.w, r.hi.x, r.hi.y, r.hi.z, r.hi.w};
  // by whole words first, then by bytes
  uint32_t a[5];
#pragma unroll
  for (int i = 0; i < 5; ++i) {
    const uint32_t s01 = off & 4 ? w[i + 1] : w[i], s23 = off & 4 ? (i + 3 < 8 ? w[i + 3] : 0u) : w[i + 2];
    a[i] = off & 8 ? s23 : s01;
  }
  const uint32_t by = 8 * (off & 3);
  const uint4 v = make_uint4(__funnelshift_r(a[0], a[1], by), __funnelshift_r(a[1], a[2], by), __funnelshift_r(a[2], a[3], by),
                             __funnelshift_r(a[3], a[4], by));
  return there < 16 ? first_bytes(v, there) : v;
}
#endif

}  // namespace ssn
