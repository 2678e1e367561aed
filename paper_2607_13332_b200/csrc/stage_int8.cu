// Products in 8-bit integers with scales per token and channel (include/agora_stage.h): quantisation and dispatch.
#include "stage_common.cuh"
#include "stage_int8.h"

#include <cmath>

namespace ssn {
namespace {

// ---- rows in 8 bits -------------------------------------------------------------------------------------------------
struct QuantArgs {
  const void *x;
  int8_t *q;
  float *scale;
  int64_t ldx, ldq, rows, cols;
};

// x / s rounded to the nearest integer, halves to even, exactly.  q = rint(x (1 / s)) is that or, where x / s lies within 2^-16 of
// a half, its neighbour.  The remainder x - q s is a multiple of half an ulp of s and not above s / 2 by more than one, so fma gives it
// without error: a q whose remainder is below s / 2 is right, and only the others are looked at again.
__device__ __forceinline__ int quantised(float x, float s, float inv) {
  float q = rintf(x * inv);
  const float e = fmaf(-q, s, x), half = 0.5f * s;
  if (e > half) q += 1.f;
  else if (e < -half) q -= 1.f;
  else if (fabsf(e) == half) q = 2.f * rintf(0.5f * (q + (e > 0.f ? 0.5f : -0.5f)));   // between q and its neighbour: the even one
  return (int)q;
}
// The same where 1 / s or the products leave the normal range
__device__ __forceinline__ int quantised_small(float x, float s) {
  return (int)fmin(fmax(rint((double)x / (double)s), -127.0), 127.0);
}
constexpr float kSmallScale = 1e-30f;

// The row's scale from its largest magnitude, 0 for a row with a value that is not finite, and an approximate reciprocal
__device__ __forceinline__ bool scale_of(float top, float &s, float &inv) {
  const bool fine = top < INFINITY;
  s = fine ? __fdiv_rn(top, 127.f) : 0.f;
  inv = __fdividef(1.f, s);
  return fine;
}
template <int WARPS> __device__ __forceinline__ float block_top(float top, float (&tops)[WARPS]) {
  for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
  if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
  __syncthreads();
  top = tops[0];
#pragma unroll
  for (int w = 1; w < WARPS; ++w) top = max_nan(top, tops[w]);
  return top;
}
// Largest magnitude of a piece
template <typename T> __device__ __forceinline__ float piece_top(const Chunk<T, 16 / (int)sizeof(T)> &v) {
  if constexpr (sizeof(T) == 4) {
    return max_nan(max_nan(fabsf(v.get(0)), fabsf(v.get(1))), max_nan(fabsf(v.get(2)), fabsf(v.get(3))));
  } else {
    const __nv_bfloat162 *w = reinterpret_cast<const __nv_bfloat162 *>(v.raw.v);
    const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(__habs2(w[0]), __habs2(w[1])), __hmax2_nan(__habs2(w[2]), __habs2(w[3])));
    return max_nan(__low2float(m), __high2float(m));
  }
}

// Rows on 16-byte boundaries: a CTA per row, which its threads hold in registers (NV pieces of 16 bytes each), so that it is read
// once and written once.  What a row costs besides its elements (the reduction, the division) bounds it together with HBM, so a
// thread has four pieces: 16384 x 4096 bf16 take 38 us (5.3 TB/s), fp32 52 (6.4).  Rows two to a CTA in turn, or a warp each, took longer.
template <typename T, int NV, int WARPS>
__global__ void __launch_bounds__(WARPS * 32) int8_quantize_rows_kernel(const QuantArgs a) {
  constexpr int E = 16 / (int)sizeof(T), kThreads = WARPS * 32;
  __shared__ float tops[WARPS];
  const int tid = threadIdx.x, cols = (int)a.cols;
  const int64_t r = blockIdx.x;
  const T *x = static_cast<const T *>(a.x) + r * a.ldx;
  pdl_enter();
  Chunk<T, E> v[NV];
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int at = (u * kThreads + tid) * E;
    if (at + E <= cols) {
      v[u].load(x + at);
    } else {
      float f[E];
#pragma unroll
      for (int i = 0; i < E; ++i) f[i] = at + i < cols ? to_f32<T>(x[at + i]) : 0.f;
      v[u].pack(f);
    }
  }
  float top = 0.f, s, inv;
#pragma unroll
  for (int u = 0; u < NV; ++u) top = max_nan(top, piece_top<T>(v[u]));
  const bool fine = scale_of(block_top(top, tops), s, inv);
  if (tid == 0) a.scale[r] = fine ? s : NAN;
  int8_t *q = a.q + r * a.ldq;
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int at = (u * kThreads + tid) * E;
    uint32_t word[E / 4];
    float far = 0.f;   // the largest remainder
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      uint32_t b[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {   // adding 1.5 * 2^23 rounds to an integer, whose low byte is q
        const float f = v[u].get(i + j), m = fmaf(f, inv, 12582912.f);
        far = fmaxf(far, fabsf(fmaf(-(m - 12582912.f), s, f)));
        b[j] = __float_as_uint(m);
      }
      word[i / 4] = s == 0.f ? 0u : __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    }
    const bool tiny = s > 0.f && s < kSmallScale;
    if (!tiny && s > 0.f && !(far < 0.5f * s)) {   // a quotient at or beside a half
#pragma unroll
      for (int i = 0; i < E; i += 4) {
        word[i / 4] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) word[i / 4] |= (uint32_t)(quantised(v[u].get(i + j), s, inv) & 255) << (8 * j);
      }
    }
    if (at + E <= cols && !tiny) {
      if constexpr (E == 8) *reinterpret_cast<uint2 *>(q + at) = make_uint2(word[0], word[1]);
      else *reinterpret_cast<uint32_t *>(q + at) = word[0];
    } else {   // a tiny scale, the row's end: one by one, from memory again
#pragma unroll 1
      for (int i = at; i < at + E && i < cols; ++i) {
        const float f = to_f32<T>(x[i]);
        q[i] = (int8_t)(s == 0.f ? 0 : s < kSmallScale ? quantised_small(f, s) : quantised(f, s, inv));
      }
    }
  }
}

// Rows of any length and place: two passes, an element at a time
constexpr int kQuantThreads = 256;
template <typename T>
__global__ void __launch_bounds__(kQuantThreads) int8_quantize_kernel(const QuantArgs a) {
  __shared__ float tops[kQuantThreads / 32];
  pdl_enter();
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *x = static_cast<const T *>(a.x) + r * a.ldx;
    float top = 0.f, s, inv;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < a.cols; i += kQuantThreads) top = max_nan(top, fabsf(to_f32<T>(x[i])));
    __syncthreads();   // the row before this one has been read from tops
    const bool fine = scale_of(block_top(top, tops), s, inv);
    if (threadIdx.x == 0) a.scale[r] = fine ? s : NAN;
    int8_t *q = a.q + r * a.ldq;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < a.cols; i += kQuantThreads) {
      const float v = to_f32<T>(x[i]);
      q[i] = (int8_t)(s == 0.f ? 0 : s < kSmallScale ? quantised_small(v, s) : quantised(v, s, inv));
    }
  }
}

template <typename T, int NV, int WARPS> cudaError_t launch_rows(const QuantArgs &a, cudaStream_t stream) {
  note_kernel(STAGE_KERNEL_QUANTIZE, NV | WARPS << 4);
  return launch_dependent(int8_quantize_rows_kernel<T, NV, WARPS>, (unsigned)a.rows, WARPS * 32, 0, stream, 1, a);
}

template <typename T> cudaError_t launch_quantize(const QuantArgs &a, cudaStream_t stream) {
  constexpr int E = 16 / (int)sizeof(T);
  const bool rows16 = aligned_to(a.x, 16) && (a.rows == 1 || a.ldx % E == 0) && aligned_to(a.q, E) && (a.rows == 1 || a.ldq % E == 0);
  const int64_t pieces = (a.cols + E - 1) / E;
  if (rows16 && pieces <= 4096 && a.rows <= 0x7fffffff) {
    if (pieces <= 128) return launch_rows<T, 2, 2>(a, stream);
    if (pieces <= 256) return launch_rows<T, 4, 2>(a, stream);
    if (pieces <= 512) return launch_rows<T, 4, 4>(a, stream);
    if (pieces <= 1024) return launch_rows<T, 4, 8>(a, stream);
    if (pieces <= 2048) return launch_rows<T, 4, 16>(a, stream);
    return launch_rows<T, 8, 16>(a, stream);
  }
  note_kernel(STAGE_KERNEL_QUANTIZE, 0);
  const int64_t cap = (int64_t)stage_sm_count() * 8;
  return launch_dependent(int8_quantize_kernel<T>, (unsigned)(a.rows < cap ? a.rows : cap), kQuantThreads, 0, stream, 1, a);
}

// ---- few tokens -------------------------------------------------------------------------------------------------------
// A warp takes kChannels output channels and all tokens: 16 bytes of a weight row per lane and step against the same 16 bytes
// of every token (out of L1).  The weights' bytes bound it; with no tensor maps and no tensor memory to set up, a call is
// shorter than the tensor-core kernels' up to kFewTokens tokens.
constexpr int kFewTokens = 2, kChannels = 2, kFewWarps = 4;
constexpr int64_t kFewBytes = 64 << 20;

template <typename T, int N, bool ANYWHERE>
__global__ void __launch_bounds__(kFewWarps * 32) int8_few_kernel(const Int8Matmul a) {
  constexpr int U = 4;   // steps in flight
  const int lane = threadIdx.x & 31;
  pdl_enter();
  const int64_t o0 = ((int64_t)blockIdx.x * kFewWarps + (threadIdx.x >> 5)) * kChannels;
  if (o0 >= a.outer) return;
  int acc[N][kChannels] = {};
  const int pieces = (int)((a.inner + 15) / 16), last = (int)(a.inner & 15);
  auto fetch = [&](const int8_t *row, int piece) {
    if (ANYWHERE) return row16(fetch_row16(row, piece * 16, (int)a.inner), row, piece * 16, (int)a.inner);
    const uint4 v = __ldg(reinterpret_cast<const uint4 *>(row) + piece);
    return piece == pieces - 1 && last != 0 ? first_bytes(v, last) : v;
  };
  for (int p0 = lane; p0 < pieces; p0 += 32 * U) {
    uint4 w[kChannels][U];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int c = 0; c < kChannels; ++c) {
        const int p = p0 + 32 * u;
        w[c][u] = make_uint4(0, 0, 0, 0);
        if (p < pieces && o0 + c < a.outer) w[c][u] = fetch(a.wq + (o0 + c) * a.ldw, p);
      }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int p = p0 + 32 * u;
      if (p >= pieces) break;
#pragma unroll
      for (int t = 0; t < N; ++t) {
        const uint4 x = fetch(a.xq + t * a.ldx, p);
#pragma unroll
        for (int c = 0; c < kChannels; ++c) {
          acc[t][c] = __dp4a((int)x.x, (int)w[c][u].x, acc[t][c]);
          acc[t][c] = __dp4a((int)x.y, (int)w[c][u].y, acc[t][c]);
          acc[t][c] = __dp4a((int)x.z, (int)w[c][u].z, acc[t][c]);
          acc[t][c] = __dp4a((int)x.w, (int)w[c][u].w, acc[t][c]);
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int c = 0; c < kChannels; ++c) {
      const int sum = __reduce_add_sync(0xffffffffu, acc[t][c]);
      if (lane == t * kChannels + c && o0 + c < a.outer)
        static_cast<T *>(a.y)[t * a.ldy + o0 + c] = from_f32<T>((float)sum * a.xs[t] * a.ws[o0 + c]);
    }
}

template <typename T, bool ANYWHERE> cudaError_t launch_few(const Int8Matmul &a, cudaStream_t stream) {
  const unsigned grid = (unsigned)((a.outer + kFewWarps * kChannels - 1) / (kFewWarps * kChannels));
  note_kernel(STAGE_KERNEL_INT8_DOT, (int)a.n | (ANYWHERE ? STAGE_KVAR_ANYWHERE : 0));
  if (a.n == 1) return launch_dependent(int8_few_kernel<T, 1, ANYWHERE>, grid, kFewWarps * 32, 0, stream, 1, a);
  return launch_dependent(int8_few_kernel<T, 2, ANYWHERE>, grid, kFewWarps * 32, 0, stream, 1, a);
}

template <typename T> cudaError_t launch_product(const Int8Matmul &a, cudaStream_t stream) {
  const bool rows16 = ((reinterpret_cast<uintptr_t>(a.xq) | reinterpret_cast<uintptr_t>(a.wq) | (uintptr_t)a.ldx | (uintptr_t)a.ldw) & 15) == 0;
  if (a.n <= kFewTokens && a.outer * a.inner <= kFewBytes) return rows16 ? launch_few<T, false>(a, stream) : launch_few<T, true>(a, stream);
  return launch_int8_umma(a, sizeof(T) == 4, rows16, stage_sm_count(), stream);
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
  if (!aligned_to(x, dtype == SSN_F32 ? 4 : 2) || !aligned_to(scale, 4)) return SSN_ERR_SHAPE;
  const QuantArgs a{x, q, scale, ldx, ldq, rows, cols};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return launched(dtype == SSN_F32 ? launch_quantize<float>(a, s) : launch_quantize<__nv_bfloat16>(a, s));
}

ssn_status_t stage_int8_matmul(const int8_t *xq, int64_t ldx, const float *xs, const int8_t *wq, int64_t ldw, const float *ws,
                               int64_t n_tokens, int64_t inner, int64_t outer, void *y, int64_t ldy, int32_t dtype,
                               int32_t *dev_status, void *stream) {
  if (dtype != SSN_F32 && dtype != SSN_BF16) return SSN_ERR_DTYPE;
  constexpr int64_t kMostRows = 0x7fffff00;   // row coordinates and tile counts are 32-bit numbers
  if (n_tokens < 0 || outer < 0 || n_tokens > kMostRows || outer > kMostRows || inner < 1 || inner > STAGE_INT8_MAX_INNER || ldx < inner || ldw < inner || ldy < outer)
    return SSN_ERR_SHAPE;
  if (n_tokens == 0 || outer == 0) return SSN_OK;
  constexpr int64_t kFar = (int64_t)1 << 60;
  if (ldx > kFar / n_tokens || ldy > kFar / n_tokens || ldw > kFar / outer || n_tokens > kFar / outer) return SSN_ERR_SHAPE;
  if (xq == nullptr || xs == nullptr || wq == nullptr || ws == nullptr || y == nullptr) return SSN_ERR_NULL;
  if (!aligned_to(y, dtype == SSN_F32 ? 4 : 2) || !aligned_to(xs, 4) || !aligned_to(ws, 4) || !aligned_to(dev_status, 4)) return SSN_ERR_SHAPE;
  const Int8Matmul given{xq, wq, xs, ws, y, ldx, ldw, ldy, n_tokens, inner, outer, dev_status};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // the pitch of a single row does not matter
  Int8Matmul a = given;
  if (a.n == 1) a.ldx = (a.inner + 15) / 16 * 16;
  if (a.outer == 1) a.ldw = (a.inner + 15) / 16 * 16;
  return launched(dtype == SSN_F32 ? launch_product<float>(a, s) : launch_product<__nv_bfloat16>(a, s));
}

}  // extern "C"
