// What the stage operators (include/agora_stage.h) share: chunked element access, launch geometry, dependent launches.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "agora_stage.h"
#include "codec_mma_launch.h"

namespace ssn {

inline bool aligned_to(const void *p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// SMs of the current device (148 when the runtime does not say)
inline int stage_sm_count() {
  static std::atomic<int> cached[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  int n = cached[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) n = 148;
    cached[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

inline ssn_status_t launched(cudaError_t e, int launches = 1) {
  if (e != cudaSuccess) {
    cudaGetLastError();
    return SSN_ERR_CUDA;
  }
  count_launches(launches);
  return SSN_OK;
}

// Every stage kernel is launched with launch_dependent: it waits for the kernel in front of it before it touches global
// memory, and lets the one behind it start its own set-up.
__device__ __forceinline__ void pdl_enter() {
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
}

// Clusters: the address of this CTA's shared memory location in the CTA of another rank; a barrier over all threads
__device__ __forceinline__ uint32_t smem_address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t map_to_rank(uint32_t addr, uint32_t rank) {
  uint32_t remote;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(remote) : "r"(addr), "r"(rank));
  return remote;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}


// V elements of T as one access of V * sizeof(T) = 2 .. 16 bytes
template <int BYTES> struct RawBytes;
template <> struct RawBytes<2> { uint16_t v[1]; };
template <> struct __align__(4) RawBytes<4> { uint32_t v[1]; };
template <> struct __align__(8) RawBytes<8> { uint32_t v[2]; };
template <> struct __align__(16) RawBytes<16> { uint32_t v[4]; };

template <typename T, int V> struct Chunk {
  RawBytes<V * (int)sizeof(T)> raw;
  __device__ __forceinline__ void load(const T *p) { raw = *reinterpret_cast<const RawBytes<V * (int)sizeof(T)> *>(p); }
  __device__ __forceinline__ void store(T *p) const { *reinterpret_cast<RawBytes<V * (int)sizeof(T)> *>(p) = raw; }
  __device__ __forceinline__ float get(int i) const;
  __device__ __forceinline__ void pack(const float (&x)[V]);
};
template <typename T, int V> __device__ __forceinline__ float Chunk<T, V>::get(int i) const {
  if constexpr (sizeof(T) == 4) {
    return __uint_as_float(raw.v[i]);
  } else if constexpr (V == 1) {
    return __uint_as_float((uint32_t)raw.v[0] << 16);
  } else {
    return __uint_as_float((i & 1) ? (raw.v[i >> 1] & 0xffff0000u) : (raw.v[i >> 1] << 16));
  }
}
template <typename T, int V> __device__ __forceinline__ void Chunk<T, V>::pack(const float (&x)[V]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < V; ++i) raw.v[i] = __float_as_uint(x[i]);
  } else if constexpr (V == 1) {
    raw.v[0] = __bfloat16_as_ushort(__float2bfloat16_rn(x[0]));
  } else {
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(x[i], x[i + 1]);
      raw.v[i >> 1] = *reinterpret_cast<const uint32_t *>(&b);
    }
  }
}

// The larger one, a NaN if either is one
__device__ __forceinline__ float max_nan(float a, float b) {
  float m;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
  return m;
}

// Two fp32 values per instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rn.f32x2 d, a, b, c;\nmov.b64 {%0, %1}, d;\n}\n"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nadd.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}\n"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmul.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}\n"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

// V values at a time, two per instruction where V is even: d = a b, d = a b + c, d = s a, d = s a + c
template <int V> __device__ __forceinline__ void v_mul(float (&d)[V], const float (&a)[V], const float (&b)[V]) {
#pragma unroll
  for (int i = 0; i + 1 < V; i += 2) {
    const float2 r = mul2({a[i], a[i + 1]}, {b[i], b[i + 1]});
    d[i] = r.x, d[i + 1] = r.y;
  }
  if constexpr (V == 1) d[0] = a[0] * b[0];
}
template <int V> __device__ __forceinline__ void v_fma(float (&d)[V], const float (&a)[V], const float (&b)[V], const float (&c)[V]) {
#pragma unroll
  for (int i = 0; i + 1 < V; i += 2) {
    const float2 r = fma2({a[i], a[i + 1]}, {b[i], b[i + 1]}, {c[i], c[i + 1]});
    d[i] = r.x, d[i + 1] = r.y;
  }
  if constexpr (V == 1) d[0] = fmaf(a[0], b[0], c[0]);
}
template <int V> __device__ __forceinline__ void v_scale(float (&d)[V], float s, const float (&a)[V]) {
#pragma unroll
  for (int i = 0; i + 1 < V; i += 2) {
    const float2 r = mul2({s, s}, {a[i], a[i + 1]});
    d[i] = r.x, d[i + 1] = r.y;
  }
  if constexpr (V == 1) d[0] = s * a[0];
}
template <int V> __device__ __forceinline__ void v_axpy(float (&d)[V], float s, const float (&a)[V], const float (&c)[V]) {
#pragma unroll
  for (int i = 0; i + 1 < V; i += 2) {
    const float2 r = fma2({s, s}, {a[i], a[i + 1]}, {c[i], c[i + 1]});
    d[i] = r.x, d[i + 1] = r.y;
  }
  if constexpr (V == 1) d[0] = fmaf(s, a[0], c[0]);
}

template <int V> __device__ __forceinline__ float v_total(const float (&a)[V]) {
  if constexpr (V == 1) return a[0];
  else if constexpr (V == 2) return a[0] + a[1];
  else {
    float h[V / 2];
#pragma unroll
    for (int i = 0; i < V / 2; i += 2) {
      const float2 r = add2({a[i], a[i + 1]}, {a[i + V / 2], a[i + 1 + V / 2]});
      h[i] = r.x, h[i + 1] = r.y;
    }
    return v_total<V / 2>(h);
  }
}

}  // namespace ssn
