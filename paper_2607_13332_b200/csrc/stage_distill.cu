// Loss of a student's logits against a teacher's top logits, with the logits' gradient (include/agora_stage.h).
//
// With m the row's largest logit and L = sum exp((s - m) / tau), everything but the teacher's entries follows from (m, L):
// the gradient is w tau exp((s - m) / tau) / L, minus w tau p at the teacher's ids.  The loss reads the row once; the
// gradient reads it once more out of L2 and writes it once, so that HBM sees the row read once and written once.
//
// What bounds it: HBM for the loss of long rows (2048 x 128256 bf16 in 100 us, 5.2 TB/s; fp32 in 186, 5.6).  The gradient (8192 x
// 128256 bf16 in 0.97 ms, 4.3 TB/s) fills neither HBM (56 % in a capture) nor the pipe of its exponentials (54 %; two per element,
// 16 lanes per clock and SM): a row is two passes with reductions between them, which the few warps that its pieces in flight leave
// room for (a third of an SM's) do not hide, and part of the second pass misses L2.  Tried and dropped: the exponentials of a row kept in the registers of a cluster of eight
// CTAs, so that each is computed once (1.44 ms: 33 of the 37 clusters fit, and 20 warps share too little of a row); a ring of
// bulk copies with a warp of its own (1.01 ms); registers filled a round ahead (fewer warps, slower); bf16 widened by shifts
// before the subtraction (1.01 against 0.96 ms with four pieces in flight); a quarter of the exponentials by a polynomial on the
// multiply-add pipe (1.04 ms).  Of 8192 rows about a third of the second pass misses L2 (444 rows of 256 KB are under way at a
// time); two CTAs per SM instead of three, with twelve pieces in flight, cost in latency what they save (0.95), as do 384 threads
// (0.96), and 512 threads take 0.91 for the gradient but 109 us for the loss.
//
// Sums are fp32 per thread, relative to the thread's running maximum, then over warps and CTAs in a fixed order; the loss
// itself, a difference of large terms, is put together in 64 bits.
#include "stage_common.cuh"

#include <cmath>

namespace ssn {
namespace {

constexpr int kMaxWarps = 8, kMaxCluster = 8;
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

// What a set of logits contributes: its maximum m and the sum of exp2((s - m) scale) over it, scale = log2(e) / tau.  The
// difference comes first: s scale - m scale in one fma is an instruction less, but loses everything where the logits are large
// (a mask of the type's lowest value).
struct MaxSum {
  float m, l;
};
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }   // for an empty set any number will do
// what turns a sum over a set of maximum m into one from another base; a set without a maximum has no sum (or a NaN)
__device__ __forceinline__ float rescale(float m, float base, float scale) {
  return m == -INFINITY ? 0.f : exp2_approx((m - base) * scale);
}
// over the lanes of a warp, in an order that does not depend on the lane
__device__ __forceinline__ MaxSum merge_warp(MaxSum ms, float scale) {
  float m = ms.m;
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float l = ms.l * rescale(ms.m, base_of(m), scale);
  for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
  return {m, l};
}

// 16 bytes of a row
template <typename T> struct Piece {
  static constexpr int E = 16 / (int)sizeof(T), kPairs = E / 2;
  Chunk<T, E> c;
  __device__ __forceinline__ void set(float v) {
    float x[E];
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = v;
    c.pack(x);
  }
  __device__ __forceinline__ void load(const void *p, bool last_use) {
    const uint4 v = last_use ? __ldcs(static_cast<const uint4 *>(p)) : *static_cast<const uint4 *>(p);
    c.raw.v[0] = v.x, c.raw.v[1] = v.y, c.raw.v[2] = v.z, c.raw.v[3] = v.w;
  }
  __device__ __forceinline__ void store(void *p) const { __stcs(static_cast<uint4 *>(p), make_uint4(c.raw.v[0], c.raw.v[1], c.raw.v[2], c.raw.v[3])); }
  // elements [first, first + E) of a row; those outside [0, vocab) are -inf, and are not written
  __device__ __forceinline__ void load_some(const T *row, int64_t first, int64_t vocab) {
    float x[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      x[i] = -INFINITY;
      if (first + i >= 0 && first + i < vocab) x[i] = to_f32<T>(row[first + i]);
    }
    c.pack(x);
  }
  __device__ __forceinline__ void store_some(T *row, int64_t first, int64_t vocab) const {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (first + i >= 0 && first + i < vocab) row[first + i] = from_f32<T>(c.get(i));   // exact: it was rounded when packed
  }
  // (s - base) scale of the pair i; a bf16 is widened by the subtraction itself
  __device__ __forceinline__ float2 exponents(int i, float base, float scale) const {
    float2 d;
    if constexpr (sizeof(T) == 2)
      asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %2;\nsub.rn.f32.bf16 %0, l, %3;\nsub.rn.f32.bf16 %1, h, %3;\n}\n" : "=f"(d.x), "=f"(d.y) : "r"(c.raw.v[i]), "f"(base));
    else
      d = add2(make_float2(c.get(2 * i), c.get(2 * i + 1)), make_float2(-base, -base));
    return mul2(d, make_float2(scale, scale));
  }
  __device__ __forceinline__ float largest() const {
    if constexpr (sizeof(T) == 4) {
      return fmaxf(fmaxf(c.get(0), c.get(1)), fmaxf(c.get(2), c.get(3)));
    } else {   // maxima of both halves of the words; like fmaxf they pass over a NaN
      const __nv_bfloat162 *w = reinterpret_cast<const __nv_bfloat162 *>(c.raw.v);
      const __nv_bfloat162 m = __hmax2(__hmax2(w[0], w[1]), __hmax2(w[2], w[3]));
      return fmaxf(__low2float(m), __high2float(m));
    }
  }
  __device__ __forceinline__ float2 sum_exp(float2 l, float base, float scale) const {
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const float2 y = exponents(i, base, scale);
      l = add2(l, make_float2(exp2_approx(y.x), exp2_approx(y.y)));
    }
    return l;
  }
  __device__ __forceinline__ void to_gradient(float base, float scale, float c_) {
    float g[E];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const float2 y = exponents(i, base, scale);
      const float2 z = mul2(make_float2(exp2_approx(y.x), exp2_approx(y.y)), make_float2(c_, c_));
      g[2 * i] = z.x;
      g[2 * i + 1] = z.y;
    }
    c.pack(g);
  }
};

// log x to 2^-25 absolutely: the exponent's part in 64 bits, the mantissa's, at most log(2) / 2 in size, by logf.  A log in 64
// bits takes a warp over a microsecond, which rows of a few microseconds would wait for.
__device__ __forceinline__ double log_of(float x) {
  if (!(x >= 1e-37f && x < INFINITY)) return (double)logf(x);
  const int32_t bits = __float_as_int(x) - 0x3f3504f3;   // 1 / sqrt(2) .. sqrt(2)
  const int32_t k = bits >> 23;
  return (double)k * 0.69314718055994531 + (double)logf(__int_as_float((bits & 0x7fffff) + 0x3f3504f3));
}

// What some of the teacher's entries contribute: their largest logit, the sum of e = exp((top - m) / tau), and the sum of
// e (top - s) over those whose column is at hand.  The quotient of the two sums is a mean of numbers that may all be large (logits are
// as good with any constant added), from which as large a one is taken: both are sums of the same fp32 terms in 64 bits, so that
// the weights of the mean add up to 1.
struct Teacher {
  float m;
  double sum, a;
};

// Resident CTAs of `threads`: what leaves the pieces in flight in registers
constexpr int per_sm(int threads, bool grad) { return threads == 256 ? (grad ? 3 : 4) : (grad ? 8 : 10); }

struct __align__(16) Part {   // one CTA's share of a row
  double a;
  MaxSum ms;
};

struct Shared {
  MaxSum ms[kMaxWarps];
  Teacher teacher[kMaxWarps];
  Part ctas[kMaxCluster];               // written once: a cluster has one row
  int32_t id[STAGE_DISTILL_MAX_TOP];    // -1: padding, or another CTA's column
  float e[STAGE_DISTILL_MAX_TOP];       // relative to the maximum of the warp that has the entry
  float at[STAGE_DISTILL_MAX_TOP];      // the student's logit there
};

// A CTA, or for few rows a cluster of them that shares a row's columns, streams through a row: once for (m, L), once more for
// the gradient, out of L2.  A row is cut at 16-byte boundaries into pieces: piece i holds the elements from i E - shift on, and
// only the first and the last piece can reach past the row; they are taken element by element, the others without a check.
// The teacher's entries, one per thread, are loaded a row ahead and the student's logits at their ids with the row's first
// pieces, so that their latency passes behind the row.
template <typename T, int kThreads, bool GRAD>
__global__ void __launch_bounds__(kThreads, per_sm(kThreads, GRAD)) distill_kernel(const __grid_constant__ DistillArgs a) {
  constexpr int E = Piece<T>::E, U = kThreads == 256 ? 6 : 4, kWarps = kThreads / 32;   // U pieces in flight per thread
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint32_t cluster, rank;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;\n" : "=r"(cluster));
  asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(rank));
  const float scale = kLog2e / a.tau, inv_tau = 1.f / a.tau;
  if (cluster > 1) cluster_sync();   // the peers have started: their shared memory may be written
  pdl_enter();
  const int64_t workers = gridDim.x / cluster;
  int next_id = -1;
  float next_top = 0.f, next_w = 1.f;
  auto look = [&](int64_t t) {
    if (t >= a.n) return;
    if (tid < a.top_k) {
      next_id = a.ids[t * a.ldi + tid];
      next_top = a.top[t * a.ldt + tid];
    }
    if (a.weight != nullptr) next_w = a.weight[t];
  };
  look(blockIdx.x / cluster);
  for (int64_t t = blockIdx.x / cluster; t < a.n; t += workers) {
    const T *row = static_cast<const T *>(a.logits) + t * a.ldl;
    T *out = GRAD ? static_cast<T *>(a.out) + t * a.ldd : nullptr;
    const int shift = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    const int pieces = (int)((shift + a.vocab + E - 1) / E), per = (pieces + (int)cluster - 1) / (int)cluster;
    const int lo = min((int)rank * per, pieces), hi = min(lo + per, pieces);
    const int in_lo = max(lo, 1), in_hi = min(hi, pieces - 1);   // without the row's first and last piece
    // the piece at the row's end that this thread takes, if any: the first one, or the last one where that is another
    const int edge = tid == 0 && lo == 0 && hi > 0 ? 0 : tid == 32 && hi == pieces && pieces > 1 && lo < hi ? pieces - 1 : -1;
    const unsigned char *src = reinterpret_cast<const unsigned char *>(row) - shift * (int)sizeof(T) + ((int64_t)in_lo + tid) * 16;
    unsigned char *dst = GRAD ? reinterpret_cast<unsigned char *>(out) - shift * (int)sizeof(T) + ((int64_t)in_lo + tid) * 16 : nullptr;
    const bool same = GRAD && ((reinterpret_cast<uintptr_t>(row) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
    const int mine = in_hi - in_lo - tid;   // pieces from this thread's first one on, every kThreads-th is its own
    const float w = next_w;

    // the teacher's entries of this thread: j = tid, tid + kThreads, ...
    __syncthreads();   // the row before this one is done with what is shared
    float tm = -INFINITY, own_at = 0.f;
    bool any = false;
    for (int j = tid; j < a.top_k; j += kThreads) {
      int32_t id = j == tid ? next_id : a.ids[t * a.ldi + j];
      const float v = j == tid ? next_top : a.top[t * a.ldt + j];
      if (id >= 0 && id < a.vocab) {
        tm = fmaxf(tm, v);
        any = any || v != -INFINITY;
      } else {
        if (id != -1 && rank == 0 && a.dev_status != nullptr) atomicOr(a.dev_status, SSN_DEV_BAD_ID);
        id = -1;
      }
      const int piece = id >= 0 ? (shift + id) / E : -1;
      const float s = piece >= lo && piece < hi ? to_f32<T>(row[id]) : 0.f;
      if (j == tid) own_at = s;   // it arrives while the row passes
      else sh.at[j] = s;
      sh.e[j] = id >= 0 ? v : -INFINITY;
      sh.id[j] = piece >= lo && piece < hi ? id : -1;
    }
    look(t + workers);
    const bool on = __syncthreads_or(any && w != 0.f);
    if (!on) {   // nothing to learn from this row
      if (tid == 0 && rank == 0) a.loss[t] = 0.f;
      if (GRAD) {
        Piece<T> z;
        z.set(0.f);
        if (same)
          for (int i = 0; i < mine; i += kThreads) z.store(dst + (int64_t)i * 16);
        else
          for (int i = 0; i < mine; i += kThreads) z.store_some(out, (int64_t)(in_lo + tid + i) * E - shift, a.vocab);
        if (edge >= 0) z.store_some(out, (int64_t)edge * E - shift, a.vocab);
      }
      continue;
    }

    float m = -INFINITY;
    float2 l = make_float2(0.f, 0.f);
    auto add = [&](Piece<T> (&x)[U]) {
      float most = m;
#pragma unroll
      for (int u = 0; u < U; ++u) most = fmaxf(most, x[u].largest());
      const float base = base_of(most), f = rescale(m, base, scale);
      l = mul2(l, make_float2(f, f));
#pragma unroll
      for (int u = 0; u < U; ++u) l = x[u].sum_exp(l, base, scale);
      m = most;
    };
    Piece<T> x[U];
    int at = 0;
    for (; at + (U - 1) * kThreads < mine; at += U * kThreads) {
#pragma unroll
      for (int u = 0; u < U; ++u) x[u].load(src + (int64_t)(at + u * kThreads) * 16, !GRAD);
      add(x);
    }
    if (at < mine || edge >= 0) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (u < U - 1 && at + u * kThreads < mine) x[u].load(src + (int64_t)(at + u * kThreads) * 16, !GRAD);
        else x[u].set(-INFINITY);
      }
      if (edge >= 0) x[U - 1].load_some(row, (int64_t)edge * E - shift, a.vocab);
      add(x);
    }
    const MaxSum own = merge_warp({m, l.x + l.y}, scale);
    if (lane == 0) sh.ms[warp] = own;
    if (warp * 32 < a.top_k) {   // the warp's entries
      if (tid < a.top_k) sh.at[tid] = own_at;
      for (int o = 16; o > 0; o >>= 1) tm = fmaxf(tm, __shfl_xor_sync(0xffffffffu, tm, o));
      double sum = 0.0, sa = 0.0;
      for (int j = tid; j < a.top_k; j += kThreads) {
        const float v = sh.e[j];
        float e = 0.f;
        if (v != -INFINITY) {   // of an entry, and one with mass
          e = expf((v - tm) * inv_tau);
          if (sh.id[j] >= 0 && !(e == 0.f)) sa += (double)e * ((double)v - (double)sh.at[j]);
        }
        sum += (double)e;
        sh.e[j] = e;
      }
      for (int o = 16; o > 0; o >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
        sa += __shfl_xor_sync(0xffffffffu, sa, o);
      }
      if (lane == 0) sh.teacher[warp] = {tm, sum, sa};
    }
    __syncthreads();
    MaxSum ms = merge_warp(lane < kWarps ? sh.ms[lane] : MaxSum{-INFINITY, 0.f}, scale);
    // the teacher's row: the warps' shares, one after the other
    const int tw = min(kWarps, (a.top_k + 31) / 32);
    float top_m = sh.teacher[0].m;
    double tsum = 0.0, ta = 0.0;
    for (int i = 1; i < tw; ++i) top_m = fmaxf(top_m, sh.teacher[i].m);
    auto share = [&](int i) { return sh.teacher[i].m == -INFINITY ? 0.f : expf((sh.teacher[i].m - top_m) * inv_tau); };
    for (int i = 0; i < tw; ++i) {
      const float f = share(i);
      tsum += sh.teacher[i].sum * (double)f;
      ta += sh.teacher[i].a * (double)f;
    }
    if (cluster > 1) {
      if (warp == 0) {
        if (lane < (int)cluster) {   // to the CTA of that rank
          const uint32_t to = map_to_rank(smem_address(&sh.ctas[rank]), (uint32_t)lane);
          asm volatile("st.shared::cluster.f64 [%0], %1;\n" ::"r"(to), "d"(ta) : "memory");
          asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};\n" ::"r"(to + 8), "f"(ms.m), "f"(ms.l) : "memory");
        }
        __syncwarp();
      }
      cluster_sync();
      ms = merge_warp(lane < (int)cluster ? sh.ctas[lane].ms : MaxSum{-INFINITY, 0.f}, scale);
      ta = 0.0;
      for (int i = 0; i < (int)cluster; ++i) ta += sh.ctas[i].a;
    }
    if (tid == 0 && rank == 0) {
      // log p = (top - top_m) / tau - log tsum, the student's log sum is m / tau + log l
      const double tau = (double)a.tau;
      const double r0 = (double)(1.f / (float)tsum), r1 = r0 * (2.0 - tsum * r0);   // 1 / tsum to 2^-45: a division in 64 bits takes long
      a.loss[t] = (float)((double)w * tau * (ta * r1 - (double)top_m + (double)ms.m + tau * (log_of(ms.l) - log_of((float)tsum))));
    }
    if (GRAD) {
      const float c = w * a.tau / ms.l, sum_p = (float)tsum;
      auto put = [&](Piece<T> &v, int i) {
        v.to_gradient(ms.m, scale, c);
        if (same) v.store(dst + (int64_t)i * 16);
        else v.store_some(out, (int64_t)(in_lo + tid + i) * E - shift, a.vocab);
      };
      // from the end: what was read last is what L2 has for certain
      at = mine > 0 ? (mine - 1) / kThreads * kThreads : -1;
      for (; at - (U - 1) * kThreads >= 0; at -= U * kThreads) {
#pragma unroll
        for (int u = 0; u < U; ++u) x[u].load(src + (int64_t)(at - u * kThreads) * 16, true);
#pragma unroll
        for (int u = 0; u < U; ++u) put(x[u], at - u * kThreads);
      }
      for (; at >= 0; at -= kThreads) {
        x[0].load(src + (int64_t)at * 16, true);
        put(x[0], at);
      }
      if (edge >= 0) {
        x[0].load_some(row, (int64_t)edge * E - shift, a.vocab);
        x[0].to_gradient(ms.m, scale, c);
        x[0].store_some(out, (int64_t)edge * E - shift, a.vocab);
      }
      __syncthreads();   // the teacher's ids are written a second time, after the row
      // by the first entry of an id, with the p of all of them: eight lanes look through the entries for one
      for (int j = tid >> 3; j < (a.top_k + 3 & ~3); j += kThreads / 8) {
        const int32_t id = j < a.top_k ? sh.id[j] : -1;
        float p = 0.f;
        bool first = true;
        if (id >= 0)
          for (int i = tid & 7; i < a.top_k; i += 8)
            if (sh.id[i] == id) {
              first = first && i >= j;
              p += sh.e[i] * share((i % kThreads) / 32);
            }
        for (int o = 4; o > 0; o >>= 1) {
          p += __shfl_xor_sync(0xffffffffu, p, o);
          first = __shfl_xor_sync(0xffffffffu, (int)first, o) != 0 && first;
        }
        if ((tid & 7) == 0 && id >= 0 && first) out[id] = from_f32<T>(exp2_approx((sh.at[j] - ms.m) * scale) * c - w * a.tau * (p / sum_p));
      }
    }
  }
}

template <typename T, int kThreads, bool GRAD> cudaError_t launch_threads(const DistillArgs &a, cudaStream_t stream) {
  const int sms = stage_sm_count();
  const int64_t cap = (int64_t)sms * per_sm(kThreads, GRAD);
  // CTAs per row: doubled while there are no more of them than SMs, and while each keeps pieces enough.  That leaves two CTAs per SM at
  // most, which are all resident, so that a cluster takes one row and no more.
  static_assert(per_sm(kThreads, GRAD) >= 2, "a cluster would take a second row");
  int cluster = 1;
  while (cluster < kMaxCluster && a.n * cluster <= sms && a.vocab / (Piece<T>::E * cluster * 2) >= 2 * kThreads) cluster *= 2;
  const int64_t workers = a.n < cap / cluster ? a.n : cap / cluster;
  note_kernel(STAGE_KERNEL_DISTILL, cluster | (kThreads == 256 ? STAGE_KVAR_MANY : 0) | (GRAD ? STAGE_KVAR_GRAD : 0));
  return launch_dependent(distill_kernel<T, kThreads, GRAD>, (unsigned)(workers * cluster), kThreads, 0, stream, cluster, a);
}

// Threads per CTA by the row's bytes: a row costs a CTA a few microseconds besides its bytes, which more CTAs per SM hide, while
// long rows want fewer of them (the second pass finds its row in L2).  0.5 GB of logits in rows of 64 / 130 / 256 KB, with the
// gradient: 128 threads 254 / 276 / 292 us, 256 threads 287 / 246 / 269; the loss alone 104 / 103 / 109 and 130 / 104 / 101.  (With six
// pieces in flight instead of four, 256 threads take another tenth off rows of 256 KB.)  Both calls add a row up in the same
// order, so that its loss is the same number with the gradient and without.
template <typename T> cudaError_t launch_distill(const DistillArgs &a, cudaStream_t stream) {
  const bool many = a.vocab * (int64_t)sizeof(T) >= 98304;
  if (a.out == nullptr) return many ? launch_threads<T, 256, false>(a, stream) : launch_threads<T, 128, false>(a, stream);
  return many ? launch_threads<T, 256, true>(a, stream) : launch_threads<T, 128, true>(a, stream);
}

}  // namespace
}  // namespace ssn

using namespace ssn;

extern "C" ssn_status_t stage_distill_loss(const void *logits, int64_t ldl, int32_t dtype, int64_t n_tokens, int64_t vocab,
                                           const int32_t *ids, int64_t ldi, const float *top, int64_t ldt, int32_t top_k,
                                           const float *weight, float tau, float *loss, void *dlogits, int64_t ldd,
                                           int32_t *dev_status, void *stream) {
  if (dtype != SSN_F32 && dtype != SSN_BF16) return SSN_ERR_DTYPE;
  if (n_tokens < 0 || vocab < 1 || vocab > 0x7ffffff0LL || top_k < 1 || top_k > STAGE_DISTILL_MAX_TOP) return SSN_ERR_SHAPE;
  if (ldl < vocab || ldi < top_k || ldt < top_k || (dlogits != nullptr && ldd < vocab)) return SSN_ERR_SHAPE;
  if (!(tau >= STAGE_DISTILL_MIN_TAU && tau <= STAGE_DISTILL_MAX_TAU)) return SSN_ERR_SHAPE;
  if (n_tokens == 0) return SSN_OK;
  const int64_t far = ((int64_t)1 << 60) / n_tokens;
  if (ldl > far || ldi > far || ldt > far || (dlogits != nullptr && ldd > far)) return SSN_ERR_SHAPE;
  if (logits == nullptr || ids == nullptr || top == nullptr || loss == nullptr) return SSN_ERR_NULL;
  const size_t item = dtype == SSN_F32 ? 4 : 2;
  if (!aligned_to(logits, item) || !aligned_to(dlogits, item)) return SSN_ERR_SHAPE;
  for (const void *p : {(const void *)ids, (const void *)top, (const void *)weight, (const void *)loss, (const void *)dev_status})
    if (!aligned_to(p, 4)) return SSN_ERR_SHAPE;
  if (dlogits == logits && ldd != ldl) return SSN_ERR_SHAPE;
  const DistillArgs a{logits, dlogits, ids, top, weight, loss, dev_status, ldl, ldd, ldi, ldt, n_tokens, vocab, top_k, tau};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return launched(dtype == SSN_F32 ? launch_distill<float>(a, s) : launch_distill<__nv_bfloat16>(a, s));
}
