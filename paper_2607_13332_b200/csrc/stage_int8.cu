// Products in 8-bit integers with scales per token and channel (include/agora_stage.h): quantisation and dispatch.
#include "stage_common.cuh"
#include "stage_int8.h"

#include <cmath>

namespace ssn {
namespace {

// ---- rows in 8 bits -------------------------------------------------------------------------------------------------
// A CTA per row, two passes (the second one out of L1): the largest magnitude, then the quotients.
constexpr int kQuantThreads = 256;

struct QuantArgs {
  const void *x;
  int8_t *q;
  float *scale;
  int64_t ldx, ldq, rows, cols;
};

// x / s rounded to the nearest integer, halves to even, exactly.  The fp32 quotient is off by less than 2^-16 here (|x / s|
// is at most 127.5), so only one that lies that near to a half can round the wrong way; fma gives the sign of x - s (n + 1/2)
// without error.
__device__ __forceinline__ int quantised(float x, float s, float inv) {
  const float y = x * inv;
  float q = rintf(y);
  if (fabsf(y - q) > 0.4999f) {
    const float n = floorf(y), side = fmaf(-s, n + 0.5f, x);
    q = side > 0.f ? n + 1.f : side < 0.f ? n : 2.f * rintf(0.5f * n + 0.25f);
  }
  return (int)fminf(fmaxf(q, -127.f), 127.f);
}
// The same where 1 / s or the products leave the normal range
__device__ __forceinline__ int quantised_small(float x, float s) {
  return (int)fmin(fmax(rint((double)x / (double)s), -127.0), 127.0);
}
constexpr float kSmallScale = 1e-30f;

template <typename T>
__global__ void __launch_bounds__(kQuantThreads) int8_quantize_kernel(const QuantArgs a) {
  __shared__ float tops[kQuantThreads / 32];
  pdl_enter();
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *x = static_cast<const T *>(a.x) + r * a.ldx;
    float top = 0.f;
    bool odd = false;   // an infinity or a NaN
    for (int64_t i = threadIdx.x; i < a.cols; i += kQuantThreads) {
      const float v = fabsf(to_f32<T>(x[i]));
      odd = odd || !(v < INFINITY);
      top = fmaxf(top, v);
    }
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    odd = __any_sync(0xffffffffu, odd);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = odd ? INFINITY : top;
    __syncthreads();
    top = tops[0];
    for (int w = 1; w < kQuantThreads / 32; ++w) top = fmaxf(top, tops[w]);
    const bool fine = top < INFINITY;
    const float s = fine ? __fdiv_rn(top, 127.f) : 0.f, inv = s > 0.f ? __frcp_rn(s) : 0.f;
    if (threadIdx.x == 0) a.scale[r] = fine ? s : NAN;
    int8_t *q = a.q + r * a.ldq;
    for (int64_t i = threadIdx.x; i < a.cols; i += kQuantThreads) {
      const float v = to_f32<T>(x[i]);
      q[i] = (int8_t)(s == 0.f ? 0 : s < kSmallScale ? quantised_small(v, s) : quantised(v, s, inv));
    }
  }
}

// ---- any alignment --------------------------------------------------------------------------------------------------
// 64 tokens x 64 channels per CTA, steps of 32 bytes of the inner dimension as 8 words, dp4a
template <typename T>
__global__ void __launch_bounds__(256) int8_general_kernel(const Int8Matmul a) {
  __shared__ int xt[64][9], wt[64][9];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int64_t tiles_o = (a.outer + 63) / 64, tiles = (a.n + 63) / 64 * tiles_o;
  pdl_enter();
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t t0 = tile / tiles_o * 64, o0 = tile % tiles_o * 64;
    int acc[4][4] = {};
    for (int64_t k0 = 0; k0 < a.inner; k0 += 32) {
      __syncthreads();
      for (int i = threadIdx.x; i < 64 * 8 * 2; i += 256) {
        const int r = (i & 511) >> 3, c = i & 7;
        const bool is_x = i < 512;
        const int64_t row = is_x ? t0 + r : o0 + r;
        const int8_t *src = is_x ? a.xq + row * a.ldx : a.wq + row * a.ldw;
        uint32_t word = 0;
        if (row < (is_x ? a.n : a.outer))
#pragma unroll
          for (int b = 0; b < 4; ++b)
            if (k0 + c * 4 + b < a.inner) word |= (uint32_t)(uint8_t)src[k0 + c * 4 + b] << (8 * b);
        (is_x ? xt : wt)[r][c] = (int)word;
      }
      __syncthreads();
#pragma unroll
      for (int c = 0; c < 8; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j] = __dp4a(xt[ty * 4 + i][c], wt[tx + 16 * j][c], acc[i][j]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t t = t0 + ty * 4 + i, o = o0 + tx + 16 * j;
        if (t < a.n && o < a.outer)
          static_cast<T *>(a.y)[t * a.ldy + o] = from_f32<T>((float)acc[i][j] * a.xs[t] * a.ws[o]);
      }
  }
}

template <typename T>
cudaError_t launch_general(const Int8Matmul &a, cudaStream_t stream) {
  const int64_t tiles = (a.n + 63) / 64 * ((a.outer + 63) / 64), cap = (int64_t)stage_sm_count() * 8;
  return launch_dependent(int8_general_kernel<T>, (unsigned)(tiles < cap ? tiles : cap), 256, 0, stream, 1, a);
}

}  // namespace
}  // namespace ssn

using namespace ssn;

extern "C" {

ssn_status_t stage_int8_quantize(const void *x, int64_t ldx, int32_t dtype, int64_t rows, int64_t cols, int8_t *q, int64_t ldq,
                                 float *scale, void *stream) {
  if (dtype != SSN_F32 && dtype != SSN_BF16) return SSN_ERR_DTYPE;
  if (rows < 0 || cols < 1 || ldx < cols || ldq < cols) return SSN_ERR_SHAPE;
  if (rows == 0) return SSN_OK;
  const int64_t far = ((int64_t)1 << 60) / rows;
  if (ldx > far || ldq > far) return SSN_ERR_SHAPE;
  if (x == nullptr || q == nullptr || scale == nullptr) return SSN_ERR_NULL;
  if (!aligned_to(x, dtype == SSN_F32 ? 4 : 2)) return SSN_ERR_SHAPE;
  const QuantArgs a{x, q, scale, ldx, ldq, rows, cols};
  const int64_t cap = (int64_t)stage_sm_count() * 8;
  const unsigned grid = (unsigned)(rows < cap ? rows : cap);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return launched(dtype == SSN_F32 ? launch_dependent(int8_quantize_kernel<float>, grid, kQuantThreads, 0, s, 1, a)
                                   : launch_dependent(int8_quantize_kernel<__nv_bfloat16>, grid, kQuantThreads, 0, s, 1, a));
}

ssn_status_t stage_int8_matmul(const int8_t *xq, int64_t ldx, const float *xs, const int8_t *wq, int64_t ldw, const float *ws,
                               int64_t n_tokens, int64_t inner, int64_t outer, void *y, int64_t ldy, int32_t dtype,
                               int32_t *dev_status, void *stream) {
  if (dtype != SSN_F32 && dtype != SSN_BF16) return SSN_ERR_DTYPE;
  if (n_tokens < 0 || outer < 0 || inner < 1 || inner > STAGE_INT8_MAX_INNER || ldx < inner || ldw < inner || ldy < outer)
    return SSN_ERR_SHAPE;
  if (n_tokens == 0 || outer == 0) return SSN_OK;
  constexpr int64_t kFar = (int64_t)1 << 60;
  if (ldx > kFar / n_tokens || ldy > kFar / n_tokens || ldw > kFar / outer || n_tokens > kFar / outer) return SSN_ERR_SHAPE;
  if (xq == nullptr || xs == nullptr || wq == nullptr || ws == nullptr || y == nullptr) return SSN_ERR_NULL;
  if (!aligned_to(y, dtype == SSN_F32 ? 4 : 2)) return SSN_ERR_SHAPE;
  const Int8Matmul a{xq, wq, xs, ws, y, ldx, ldw, ldy, n_tokens, inner, outer, dev_status};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = launch_int8_umma(a, dtype == SSN_F32, stage_sm_count(), s);
  if (e != cudaErrorNotSupported) return launched(e);
  return launched(dtype == SSN_F32 ? launch_general<float>(a, s) : launch_general<__nv_bfloat16>(a, s));
}

}  // extern "C"
