// Loss of a student's logits against a teacher's top logits, with the logits' gradient (include/agora_stage.h).
//
// With m the row's largest logit and L = sum exp((s - m) / tau), everything but the teacher's entries follows from (m, L):
// the gradient is w tau exp((s - m) / tau) / L, minus w tau p at the teacher's ids.  The loss reads the row once; the
// gradient reads and writes it once.
//
// Rows are taken 16 bytes at a time from the 16-byte boundary at or before their start (a vocabulary may be odd), the first
// and last piece element by element.  Sums are fp32 per thread, at most a few dozen terms relative to the thread's own
// maximum, then over warps and CTAs in a fixed order; the loss itself, a difference of large terms, is put together in 64 bits.
#include "stage_common.cuh"

#include <cmath>

namespace ssn {
namespace {

constexpr int kMaxThreads = 512, kMaxWarps = kMaxThreads / 32;
constexpr float kLog2e = 1.4426950408889634f;

struct DistillArgs {
  const void *logits;
  void *out;                // gradient or nullptr
  const int32_t *ids;
  const float *top, *weight;
  float *loss;
  int32_t *dev_status;
  int64_t ldl, ldd, ldi, ldt, n, vocab;
  int32_t top_k;
  float tau;
};

__device__ __forceinline__ float exp2_approx(float x) {   // 2 ulp; a probability below 2^-126 is 0
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// What a set of logits contributes: its maximum and the sum of exp2((s - m) scale) over it
struct MaxSum {
  float m, l;
};
__device__ __forceinline__ MaxSum merge(MaxSum a, MaxSum b, float scale) {
  const float m = fmaxf(a.m, b.m), at = m == -INFINITY ? 0.f : m;   // two empty sets stay empty
  return {m, a.l * exp2_approx((a.m - at) * scale) + b.l * exp2_approx((b.m - at) * scale)};
}

template <typename T> struct Piece {   // 16 bytes of a row
  static constexpr int E = 16 / (int)sizeof(T);
  Chunk<T, E> c;
  // elements [first, first + E) of the row; those outside [0, vocab) are -inf
  __device__ __forceinline__ void load(const T *row, int64_t first, int64_t vocab) {
    if (first >= 0 && first + E <= vocab) {
      const uint4 v = *reinterpret_cast<const uint4 *>(row + first);
      c.raw.v[0] = v.x, c.raw.v[1] = v.y, c.raw.v[2] = v.z, c.raw.v[3] = v.w;
    } else {
      float x[E];
#pragma unroll
      for (int i = 0; i < E; ++i) {
        x[i] = -INFINITY;
        if (first + i >= 0 && first + i < vocab) x[i] = to_f32<T>(row[first + i]);
      }
      c.pack(x);
    }
  }
  __device__ __forceinline__ void store(T *row, int64_t first, int64_t vocab, bool whole) const {
    if (whole && first >= 0 && first + E <= vocab) {
      *reinterpret_cast<uint4 *>(row + first) = make_uint4(c.raw.v[0], c.raw.v[1], c.raw.v[2], c.raw.v[3]);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (first + i >= 0 && first + i < vocab) row[first + i] = from_f32<T>(c.get(i));   // exact: it was rounded when packed
    }
  }
  __device__ __forceinline__ float largest() const {
    float m = c.get(0);
#pragma unroll
    for (int i = 1; i < E; ++i) m = fmaxf(m, c.get(i));
    return m;
  }
  __device__ __forceinline__ float sum_exp(float m, float scale) const {
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) l += exp2_approx((c.get(i) - m) * scale);
    return l;
  }
};

struct Shared {
  double a[kMaxWarps], p[kMaxWarps];
  MaxSum ms[kMaxWarps];
  int32_t id[STAGE_DISTILL_MAX_TOP];    // -1: padding
  float e[STAGE_DISTILL_MAX_TOP];       // exp((top - max) / tau), to be divided by their sum
  float at[STAGE_DISTILL_MAX_TOP];      // the student's logit there
};

// One CTA per row, which streams through it: once for (m, L), once more for the gradient.
template <typename T, bool GRAD>
__global__ void __launch_bounds__(kMaxThreads) distill_stream_kernel(const __grid_constant__ DistillArgs a) {
  constexpr int E = 16 / (int)sizeof(T), kUnroll = 4;
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads >> 5;
  const float scale = kLog2e / a.tau;
  pdl_enter();
  for (int64_t t = blockIdx.x; t < a.n; t += gridDim.x) {
    const float w = a.weight != nullptr ? a.weight[t] : 1.f;
    const T *row = static_cast<const T *>(a.logits) + t * a.ldl;
    T *out = GRAD ? static_cast<T *>(a.out) + t * a.ldd : nullptr;
    const int shift = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    const bool whole = GRAD && ((reinterpret_cast<uintptr_t>(row) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
    const int64_t pieces = (shift + a.vocab + E - 1) / E;

    // the teacher's maximum and sum, by every warp for itself
    const int32_t *ids = a.ids + t * a.ldi;
    const float *top = a.top + t * a.ldt;
    float tm = -INFINITY;
    bool any = false;
    for (int j = lane; j < a.top_k; j += 32) {
      const int32_t id = ids[j];
      const float x = top[j];
      if (id >= 0 && id < a.vocab) {
        tm = fmaxf(tm, x);
        any = any || x != -INFINITY;
      } else if (id != -1 && warp == 0 && a.dev_status != nullptr) {
        atomicOr(a.dev_status, SSN_DEV_BAD_ID);
      }
    }
    for (int o = 16; o > 0; o >>= 1) tm = fmaxf(tm, __shfl_xor_sync(0xffffffffu, tm, o));
    any = __any_sync(0xffffffffu, any);
    if (w == 0.f || !any) {   // nothing to learn from this row
      if (tid == 0) a.loss[t] = 0.f;
      if (GRAD) {
        const float zero[E] = {};
        Piece<T> z;
        z.c.pack(zero);
        for (int64_t i = tid; i < pieces; i += threads) z.store(out, i * E - shift, a.vocab, whole);
      }
      continue;
    }
    const float inv_tau = 1.f / a.tau;
    float tsum = 0.f;
    for (int j = lane; j < a.top_k; j += 32) {
      const int32_t id = ids[j];
      if (id >= 0 && id < a.vocab) tsum += expf((top[j] - tm) * inv_tau);
    }
    for (int o = 16; o > 0; o >>= 1) tsum += __shfl_xor_sync(0xffffffffu, tsum, o);
    __syncthreads();   // the row before this one is done with what is shared
    double part_a = 0.0, part_p = 0.0;   // sum p (log p - x), sum p
    for (int j = tid; j < a.top_k; j += threads) {
      int32_t id = ids[j];
      if (id < 0 || id >= a.vocab) id = -1;
      float e = 0.f, at = 0.f;
      if (id >= 0) {
        at = to_f32<T>(row[id]);
        e = expf((top[j] - tm) * inv_tau);
        const float p = e / tsum;
        if (!(p == 0.f)) {
          part_a += (double)p * (((double)top[j] - (double)tm - (double)at) / (double)a.tau - log((double)tsum));
          part_p += (double)p;
        }
      }
      sh.id[j] = id;
      sh.e[j] = e;
      sh.at[j] = at;
    }

    MaxSum ms{-INFINITY, 0.f};
    for (int64_t i0 = tid; i0 < pieces; i0 += (int64_t)threads * kUnroll) {
      Piece<T> x[kUnroll];
      float m = ms.m;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) x[u].load(row, (i0 + (int64_t)u * threads) * E - shift, a.vocab);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) m = fmaxf(m, x[u].largest());
      const float at = m == -INFINITY ? 0.f : m;
      float l = ms.l * exp2_approx((ms.m - at) * scale);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) l += x[u].sum_exp(at, scale);
      ms = {m, l};
    }
    for (int o = 16; o > 0; o >>= 1) {
      const MaxSum other{__shfl_xor_sync(0xffffffffu, ms.m, o), __shfl_xor_sync(0xffffffffu, ms.l, o)};
      ms = lane & o ? merge(other, ms, scale) : merge(ms, other, scale);
      part_a += __shfl_xor_sync(0xffffffffu, part_a, o);
      part_p += __shfl_xor_sync(0xffffffffu, part_p, o);
    }
    if (lane == 0) {
      sh.ms[warp] = ms;
      sh.a[warp] = part_a;
      sh.p[warp] = part_p;
    }
    __syncthreads();
    ms = sh.ms[0];
    for (int i = 1; i < warps; ++i) ms = merge(ms, sh.ms[i], scale);
    if (tid == 0) {
      double sa = 0.0, sp = 0.0;
      for (int i = 0; i < warps; ++i) sa += sh.a[i], sp += sh.p[i];
      const double lse = (double)ms.m / (double)a.tau + log((double)ms.l);
      a.loss[t] = (float)((double)w * (double)a.tau * (double)a.tau * (sa + sp * lse));
    }
    if (GRAD) {
      const float c = w * a.tau / ms.l;
      for (int64_t i = tid; i < pieces; i += threads) {
        Piece<T> x;
        x.load(row, i * E - shift, a.vocab);
        float g[E];
#pragma unroll
        for (int q = 0; q < E; ++q) g[q] = exp2_approx((x.c.get(q) - ms.m) * scale) * c;
        x.c.pack(g);
        x.store(out, i * E - shift, a.vocab, whole);
      }
      __syncthreads();   // the teacher's ids are written a second time, after the row
      for (int j = tid; j < a.top_k; j += threads) {
        const int32_t id = sh.id[j];
        if (id < 0) continue;
        float p = 0.f;
        bool first = true;
        for (int i = 0; i < a.top_k; ++i)
          if (sh.id[i] == id) {
            first = first && i >= j;
            p += sh.e[i];
          }
        if (first) out[id] = from_f32<T>(exp2_approx((sh.at[j] - ms.m) * scale) * c - w * a.tau * (p / tsum));
      }
    }
  }
}

template <typename T>
cudaError_t launch_distill(const DistillArgs &a, cudaStream_t stream) {
  const int64_t cap = (int64_t)stage_sm_count() * 4;
  const unsigned grid = (unsigned)(a.n < cap ? a.n : cap);
  if (a.out != nullptr) return launch_dependent(distill_stream_kernel<T, true>, grid, kMaxThreads, 0, stream, 1, a);
  return launch_dependent(distill_stream_kernel<T, false>, grid, kMaxThreads, 0, stream, 1, a);
}

}  // namespace
}  // namespace ssn

using namespace ssn;

extern "C" ssn_status_t stage_distill_loss(const void *logits, int64_t ldl, int32_t dtype, int64_t n_tokens, int64_t vocab,
                                           const int32_t *ids, int64_t ldi, const float *top, int64_t ldt, int32_t top_k,
                                           const float *weight, float tau, float *loss, void *dlogits, int64_t ldd,
                                           int32_t *dev_status, void *stream) {
  if (dtype != SSN_F32 && dtype != SSN_BF16) return SSN_ERR_DTYPE;
  if (n_tokens < 0 || vocab < 1 || vocab > 0x7fffffffLL || top_k < 1 || top_k > STAGE_DISTILL_MAX_TOP) return SSN_ERR_SHAPE;
  if (ldl < vocab || ldi < top_k || ldt < top_k || (dlogits != nullptr && ldd < vocab)) return SSN_ERR_SHAPE;
  if (!(tau >= STAGE_DISTILL_MIN_TAU && tau <= STAGE_DISTILL_MAX_TAU)) return SSN_ERR_SHAPE;
  if (n_tokens == 0) return SSN_OK;
  const int64_t far = ((int64_t)1 << 60) / n_tokens;
  if (ldl > far || ldi > far || ldt > far || (dlogits != nullptr && ldd > far)) return SSN_ERR_SHAPE;
  if (logits == nullptr || ids == nullptr || top == nullptr || loss == nullptr) return SSN_ERR_NULL;
  const size_t item = dtype == SSN_F32 ? 4 : 2;
  if (!aligned_to(logits, item) || !aligned_to(dlogits, item)) return SSN_ERR_SHAPE;
  if (dlogits == logits && ldd != ldl) return SSN_ERR_SHAPE;
  const DistillArgs a{logits, dlogits, ids, top, weight, loss, dev_status, ldl, ldd, ldi, ldt, n_tokens, vocab, top_k, tau};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return launched(dtype == SSN_F32 ? launch_distill<float>(a, s) : launch_distill<__nv_bfloat16>(a, s));
}
