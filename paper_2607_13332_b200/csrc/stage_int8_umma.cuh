// tcgen05 kernel of the 8-bit product (include/agora_stage.h): y = (xq wq^T) scaled by token and channel.
//
// Tiles of A rows x B rows with the sums in 32-bit integers in tensor memory (kind::i8).  A is the operand on the MMA's M side:
//   CG = 2, !SWAP   A = tokens, B = channels.  Two CTAs share a tile of 256 tokens x BN channels: each holds 128 tokens and BN / 2
//                   channels per stage, so that a byte loaded feeds twice the products of a single CTA's tile.
//   CG = 1, SWAP    A = channels, B = tokens, for few tokens: 128 channels x BN tokens.  The weights stream past once; with fewer
//                   tiles than SMs a cluster splits the inner dimension and adds its partial sums through distributed shared
//                   memory (integers: any order gives the same sum).
//
//   CG = 1, !SWAP   A = tokens, B = channels, a CTA by itself: sizes whose tiles of pairs would leave many SMs out.
//
//   warp 0     producer: per stage of 128 bytes of the inner dimension one TMA box of A and one of B, 128-byte swizzled; the
//              inner dimension's tail and rows past the end are filled with zeros, which add nothing
//   warp 1     MMA issuer (of the pair's first CTA), four K steps of 32 bytes per stage
//   warps 4-7  epilogue: tcgen05.ld of the 32 lanes each may read, scaling, stores; two accumulators, so that a tile's
//              epilogue runs behind the next tile's MMAs
//   8 more     (RAGGED: rows off 16-byte boundaries, which TMA cannot fetch) load and shift them into the stages instead
#pragma once

#include <cuda.h>

#include "codec_umma.cuh"
#include "stage_common.cuh"
#include "stage_int8.h"

namespace ssn {

struct Int8Maps {
  CUtensorMap a, b;
};

struct Int8Args {
  const float *sa, *sb;   // scales of A's and B's rows
  void *y;
  int64_t ldy;
  int32_t rows_a, rows_b, steps, tiles_a, tiles_b;   // steps of kInt8Step bytes
  const int8_t *a, *b;                               // the operands, for loads that TMA cannot do
  int64_t lda, ldb;
  int32_t inner;
  int32_t *dev_status;
};

constexpr int kInt8Step = 128, kInt8Loaders = 256;

template <int CG, int BN, bool SWAP, bool RAGGED> struct Int8Config {
  static_assert(CG == 1 || !RAGGED, "pairs of CTAs fetch by TMA");
  static constexpr int kFirstLoader = 256, kThreads = kFirstLoader + (RAGGED ? kInt8Loaders : 0);
  static constexpr int kABytes = 128 * kInt8Step, kBRows = BN / CG, kBBytes = kBRows * kInt8Step;
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kOutBytes = SWAP ? 0 : 4 * (4096 + BN * 4);   // per epilogue warp a 32 x 128-byte block of the output, and B's scales
  static constexpr int kBudget = 222 * 1024 - kOutBytes;
  static constexpr int kFit = kBudget / kStageBytes, kStages = kFit < 10 ? kFit : 10;
  static constexpr int kBars = 2 * kStages + 5;
  static constexpr int kSmemBytes = 1024 + kStages * kStageBytes + kOutBytes + kBars * 8 + 16;
  static constexpr int kTmemCols = 2 * BN < 32 ? 32 : 2 * BN;
  static_assert(kTmemCols <= 512 && (kTmemCols & (kTmemCols - 1)) == 0 && kSmemBytes <= 227 * 1024, "tile too large");
  static_assert(kBBytes % 1024 == 0, "stages start on swizzle blocks");
  // signed 8-bit A and B (both K-major), 32-bit integer sums
  static constexpr uint32_t kIdesc = (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)((128 * CG) >> 4) << 24);
};

template <int CG> __device__ __forceinline__ void int8_tma(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1) {
  if constexpr (CG == 2)   // bar: a shared::cluster address, the barrier of the pair's first CTA
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];\n"
        ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1) : "memory");
  else
    tma_load_2d(dst, map, bar, c0, c1);
}
template <int CG>
__device__ __forceinline__ void int8_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (CG == 2)
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n}\n"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
  else
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n}\n"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// Arrives on the barrier (on both CTAs' for a pair, or on those of `ranks`) when every MMA issued so far is done
template <int CG> __device__ __forceinline__ void int8_commit(uint32_t bar, uint16_t ranks = 3) {
  if constexpr (CG == 2)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n"
                 ::"r"(bar), "h"(ranks) : "memory");
  else
    umma_commit(bar);
}
// A wait of whole warps: all lanes go on, or all of them give up, since what follows it takes a converged warp
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity)); }

template <int CG, int BN, bool SWAP, bool RAGGED, typename T>
__global__ void __launch_bounds__((Int8Config<CG, BN, SWAP, RAGGED>::kThreads), 1)
int8_umma_kernel(const Int8Args a, const __grid_constant__ Int8Maps maps) {
  using Cfg = Int8Config<CG, BN, SWAP, RAGGED>;
  constexpr int S = Cfg::kStages;
  extern __shared__ __align__(128) unsigned char smem_raw[];
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t smem0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t out0 = smem0 + S * Cfg::kStageBytes, bars = out0 + Cfg::kOutBytes;
  auto full_bar = [&](int s) { return bars + s * 8; };
  auto empty_bar = [&](int s) { return bars + (S + s) * 8; };
  auto acc_full_bar = [&](int b) { return bars + (2 * S + b) * 8; };
  auto acc_empty_bar = [&](int b) { return bars + (2 * S + 2 + b) * 8; };
  const uint32_t drain_bar = bars + (2 * S + 4) * 8, tmem_slot = bars + Cfg::kBars * 8;
  volatile uint32_t *tmem_slot_ptr = reinterpret_cast<volatile uint32_t *>(smem_raw + (tmem_slot - smem_u32(smem_raw)));
  uint32_t cluster, rank;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;\n" : "=r"(cluster));
  asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(rank));

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(full_bar(s), RAGGED ? kInt8Loaders / 32 : 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(acc_full_bar(b), 1);
      mbar_init(acc_empty_bar(b), 4 * CG);
    }
    mbar_init(drain_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  if (warp == 2) {
    if constexpr (CG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(tmem_slot), "r"(Cfg::kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(tmem_slot), "r"(Cfg::kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  cluster_sync();   // the peers' barriers exist
  asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
  const uint32_t tmem_base = *tmem_slot_ptr;
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  // A role that gives up on a wait leaves its loop; the others' waits run out in turn, and every thread reaches the end.
  bool dead = false;
  auto timed_out = [&]() {
    dead = true;
    if (a.dev_status) atomicOr(a.dev_status, SSN_DEV_TIMEOUT);
  };

  // Tiles: pairs (CG = 2) or CTAs take them in turn.  A splitting cluster (CG = 1) has one tile and a range of steps per CTA.
  const int64_t tiles = (int64_t)a.tiles_a * a.tiles_b;
  const int workers = (int)(gridDim.x / cluster), worker = (int)(blockIdx.x / cluster);
  const int split = CG == 1 ? (int)cluster : 1;
  const int step_lo = (int)((int64_t)a.steps * (CG == 1 ? (int)rank : 0) / split);
  const int step_hi = (int)((int64_t)a.steps * (CG == 1 ? (int)rank + 1 : 1) / split);
  // Eight A tiles go with a B tile before the next B tile: the tiles that run at one time share rows in L2.
  constexpr int kGroup = 8;
  auto place = [&](int64_t tile, int &ta, int &tb) {
    const int64_t per = (int64_t)kGroup * a.tiles_b, g = tile / per, in = tile - g * per;
    const int first = (int)(g * kGroup), wide = min(kGroup, a.tiles_a - first);
    ta = first + (int)(in % wide);
    tb = (int)(in / wide);
  };

  uint32_t v[BN <= 64 ? BN : 1];   // a splitting CTA's partial sums
  if (RAGGED && threadIdx.x >= Cfg::kFirstLoader) {
    // Loader warps: 16 bytes per lane and piece, eight lanes to a row's 128 bytes, into the layout that TMA would write
    const int loader = threadIdx.x - Cfg::kFirstLoader, piece = loader & 7, row0 = loader >> 3;
    constexpr int kRowStep = kInt8Loaders / 8, kRows = 128 + Cfg::kBRows, kPerThread = (kRows + kRowStep - 1) / kRowStep;
    int slot = 0;
    uint32_t parity = 1;
    for (int64_t tile = worker; tile < tiles && !dead; tile += workers) {
      int ta, tb;
      place(tile, ta, tb);
      Row16 next[kPerThread];
      auto row_of = [&](int i, int &bytes) {   // row i of this thread; one past the operand's end has no bytes
        const int r = row0 + i * kRowStep;
        const bool is_a = r < 128;
        const int64_t row = is_a ? (int64_t)ta * 128 + r : (int64_t)tb * BN + r - 128;
        const bool there = r < kRows && row < (is_a ? a.rows_a : a.rows_b);
        bytes = there ? a.inner : 0;
        return (is_a ? a.a : a.b) + (there ? row : 0) * (is_a ? a.lda : a.ldb);
      };
      auto fetch = [&](int st) {
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
          int bytes;
          const int8_t *row = row_of(i, bytes);
          next[i] = fetch_row16(row, st * kInt8Step + piece * 16, a.inner);
        }
      };
      fetch(step_lo);
      for (int st = step_lo; st < step_hi; ++st) {
        uint4 v[kPerThread];
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
          int bytes;
          const int8_t *row = row_of(i, bytes);
          v[i] = row16(next[i], row, st * kInt8Step + piece * 16, bytes);
        }
        if (st + 1 < step_hi) fetch(st + 1);   // on its way while this one is stored
        if (!mbar_wait_warp(empty_bar(slot), parity)) {
          timed_out();
          break;
        }
        const uint32_t base = smem0 + (uint32_t)slot * Cfg::kStageBytes;
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
          const int r = row0 + i * kRowStep;   // B's rows follow A's: both start on swizzle blocks
          if (r < kRows)
            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};\n" ::"r"(base + r * 128 + ((piece ^ (r & 7)) << 4)), "r"(v[i].x), "r"(v[i].y),
                         "r"(v[i].z), "r"(v[i].w) : "memory");
        }
        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(full_bar(slot));
        if (++slot == S) {
          slot = 0;
          parity ^= 1u;
        }
      }
    }
    __syncwarp();
  } else if (warp == 0) {
    int slot = 0, issued = 0;
    uint32_t parity = 1;
    if (!RAGGED && lane == 0) {
      for (int64_t tile = worker; tile < tiles && !dead; tile += workers) {
        int ta, tb;
        place(tile, ta, tb);
        const int row_a = (ta * CG + (CG == 2 ? (int)rank : 0)) * 128, row_b = tb * BN + (CG == 2 ? (int)rank * Cfg::kBRows : 0);
        for (int st = step_lo; st < step_hi; ++st) {
          if (!mbar_wait(empty_bar(slot), parity)) {
            timed_out();
            break;
          }
          const uint32_t base = smem0 + (uint32_t)slot * Cfg::kStageBytes;
          const uint32_t bar = CG == 2 ? map_to_rank(full_bar(slot), 0) : full_bar(slot);
          if (CG == 1 || rank == 0) mbar_expect_tx(full_bar(slot), CG * Cfg::kStageBytes);
          int8_tma<CG>(base, &maps.a, bar, st * kInt8Step, row_a);
          int8_tma<CG>(base + Cfg::kABytes, &maps.b, bar, st * kInt8Step, row_b);
          ++issued;
          if (++slot == S) {
            slot = 0;
            parity ^= 1u;
          }
        }
      }
      // No copy may land after the CTA has left, whoever gave up (the MMAs have waited for all of them if nobody did).  A pair's
      // copies, its second CTA's too, arrive on the first CTA's barriers.
      if (CG == 1 || rank == 0 || dead) {
        for (int i = 0; i < S && i < issued; ++i) {
          const int n = issued - 1 - i;
          mbar_wait(full_bar(n % S), (uint32_t)((n / S) & 1));
        }
      }
    }
    __syncwarp();
  } else if (warp == 1 && (CG == 1 || rank == 0)) {
    if (lane == 0) {
      const uint64_t desc = umma_desc(0, 16, 1024, 2);   // K-major, 128-byte swizzle, 8-row groups 1024 bytes apart
      int slot = 0, count = 0;
      uint32_t parity = 0;
      for (int64_t tile = worker; tile < tiles && !dead; tile += workers, ++count) {
        const int buf = count & 1;
        if (!mbar_wait_cluster(acc_empty_bar(buf), (uint32_t)(((count >> 1) & 1) ^ 1))) {
          timed_out();
          break;
        }
        asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
        const uint32_t d = tmem_base + (uint32_t)(buf * BN);
        for (int st = step_lo; st < step_hi; ++st) {
          if (!mbar_wait(full_bar(slot), parity)) {
            timed_out();
            break;
          }
          asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
          const uint32_t base = smem0 + (uint32_t)slot * Cfg::kStageBytes;
          const uint64_t da = desc + umma_desc_addr(base), db = desc + umma_desc_addr(base + Cfg::kABytes);
#pragma unroll
          for (int j = 0; j < kInt8Step / 32; ++j) int8_mma<CG>(d, da + j * 2, db + j * 2, Cfg::kIdesc, (st > step_lo || j > 0) ? 1u : 0u);
          int8_commit<CG>(empty_bar(slot));
          if (++slot == S) {
            slot = 0;
            parity ^= 1u;
          }
        }
        if (!dead) int8_commit<CG>(acc_full_bar(buf));
      }
      int8_commit<CG>(drain_bar, 1);   // and no MMA may be under way then: the epilogue waits for them too, unless it gave up
      mbar_wait(drain_bar, 0);
    }
    __syncwarp();
  } else if (warp >= 4 && threadIdx.x < Cfg::kFirstLoader) {
    const int quarter = warp & 3;
    const uint32_t scales = out0 + 4 * 4096 + (uint32_t)quarter * BN * 4;   // !SWAP
    int count = 0;
    for (int64_t tile = worker; tile < tiles && !dead; tile += workers, ++count) {
      int ta, tb;
      place(tile, ta, tb);
      const int buf = count & 1;
      // the scales, while the sums are still being made
      const int64_t row_a0 = (int64_t)(ta * CG + (CG == 2 ? (int)rank : 0)) * 128 + quarter * 32, row_a = row_a0 + lane;
      const int64_t row_b0 = (int64_t)tb * BN;
      const float sa = row_a < a.rows_a ? __ldg(a.sa + row_a) : 0.f;
      float tokens[SWAP ? (BN + 31) / 32 : 1];
      if constexpr (SWAP) {
#pragma unroll
        for (int i = 0; i < (BN + 31) / 32; ++i) tokens[i] = row_b0 + i * 32 + lane < a.rows_b ? __ldg(a.sb + row_b0 + i * 32 + lane) : 0.f;
      } else {
#pragma unroll
        for (int i = 0; i < BN / 32; ++i) {
          const float f = row_b0 + i * 32 + lane < a.rows_b ? __ldg(a.sb + row_b0 + i * 32 + lane) : 0.f;
          asm volatile("st.shared.f32 [%0], %1;\n" ::"r"(scales + (uint32_t)(i * 32 + lane) * 4), "f"(f) : "memory");
        }
        __syncwarp();
      }
      if (!mbar_wait_warp(acc_full_bar(buf), (uint32_t)((count >> 1) & 1))) {
        timed_out();
        break;
      }
      asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * BN);
      T *y = static_cast<T *>(a.y);
      if constexpr (SWAP) {
        // lane = channel, column = token: a warp stores 32 neighbouring channels of a token at a time
        if (split > 1) {
          if constexpr (BN <= 64) {
#pragma unroll
            for (int q = 0; q < BN / 16; ++q) {
              uint32_t w[16];
              tmem_ld16(taddr + q * 16, w);
#pragma unroll
              for (int i = 0; i < 16; ++i) v[q * 16 + i] = w[i];
            }
            asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
          }
          break;   // one tile: the sums meet below
        }
#pragma unroll
        for (int q = 0; q < BN / 16; ++q) {
          if (row_b0 + q * 16 >= a.rows_b) break;
          uint32_t w[16];
          tmem_ld16(taddr + q * 16, w);
          asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int64_t t = row_b0 + q * 16 + i;
            const float sb = __shfl_sync(0xffffffffu, tokens[q >> 1], (q & 1) * 16 + i);
            if (t < a.rows_b && row_a < a.rows_a) y[t * a.ldy + row_a] = from_f32<T>((float)(int)w[i] * sb * sa);
          }
        }
      } else {
        // lane = token, column = channel: blocks of 32 tokens x 128 bytes are turned in shared memory, rows 16 bytes at a time
        constexpr int kCols = 128 / (int)sizeof(T), kPiece = 16 / (int)sizeof(T), kTogether = 16;
        const uint32_t block = out0 + (uint32_t)quarter * 4096;
        const bool wide = ((reinterpret_cast<uintptr_t>(a.y) | (uintptr_t)(a.ldy * (int64_t)sizeof(T))) & 15) == 0;
#pragma unroll 1
        for (int c0 = 0; c0 < BN; c0 += kCols) {
          const int64_t col0 = row_b0 + c0;
          if (col0 >= a.rows_b) break;
          const bool inside = col0 + kCols <= a.rows_b;
#pragma unroll
          for (int h = 0; h < kCols / 32; ++h) {
            uint32_t w0[16], w1[16];
            tmem_ld16(taddr + c0 + h * 32, w0);
            tmem_ld16(taddr + c0 + h * 32 + 16, w1);
            asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
#pragma unroll
            for (int p = 0; p < 32 / kPiece; ++p) {
              float f[kPiece], sb[kPiece];
#pragma unroll
              for (int i = 0; i < kPiece; i += 4)
                asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];\n" : "=f"(sb[i]), "=f"(sb[i + 1]), "=f"(sb[i + 2]), "=f"(sb[i + 3])
                             : "r"(scales + (uint32_t)(c0 + h * 32 + p * kPiece + i) * 4));
#pragma unroll
              for (int i = 0; i < kPiece; ++i) {
                const int c = p * kPiece + i;
                f[i] = (float)(int)(c < 16 ? w0[c & 15] : w1[c & 15]) * sa * sb[i];
              }
              Chunk<T, kPiece> o;
              o.pack(f);
              const int piece = h * (32 / kPiece) + p;
              asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};\n" ::"r"(block + lane * 128 + ((piece ^ (lane & 7)) << 4)), "r"(o.raw.v[0]),
                           "r"(o.raw.v[1]), "r"(o.raw.v[2]), "r"(o.raw.v[3]) : "memory");
            }
          }
          __syncwarp();
          if (wide && inside) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int r = i * 4 + (lane >> 3), piece = lane & 7;
              uint4 o;
              asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];\n" : "=r"(o.x), "=r"(o.y), "=r"(o.z), "=r"(o.w)
                           : "r"(block + r * 128 + ((piece ^ (r & 7)) << 4)));
              if (row_a0 + r < a.rows_a) *reinterpret_cast<uint4 *>(y + (row_a0 + r) * a.ldy + col0 + piece * kPiece) = o;
            }
          } else {
            // rows off 16-byte boundaries: an element per lane, sixteen rows on their way at a time (with four, 4096 x 4096 x 32003 in
            // fp32 took 531 us instead of 377, and 341 with rows on boundaries)
            const int rows = (int)min((int64_t)32, a.rows_a - row_a0), cols = (int)min((int64_t)kCols, a.rows_b - col0);
            T *to = y + row_a0 * a.ldy + col0 + lane;
#pragma unroll 1
            for (int r0 = 0; r0 < 32; r0 += kTogether) {
              T o[kTogether][kCols / 32];
#pragma unroll
              for (int r = 0; r < kTogether; ++r)
#pragma unroll
                for (int h = 0; h < kCols / 32; ++h) {
                  const int at = (h * 32 + lane) * (int)sizeof(T);
                  const uint32_t src = block + (r0 + r) * 128 + (((at >> 4) ^ ((r0 + r) & 7)) << 4) + (at & 15);
                  if constexpr (sizeof(T) == 4) {
                    asm volatile("ld.shared.f32 %0, [%1];\n" : "=f"(o[r][h]) : "r"(src));
                  } else {
                    unsigned short bits;
                    asm volatile("ld.shared.u16 %0, [%1];\n" : "=h"(bits) : "r"(src));
                    o[r][h] = __ushort_as_bfloat16(bits);
                  }
                }
#pragma unroll
              for (int r = 0; r < kTogether; ++r) {
#pragma unroll
                for (int h = 0; h < kCols / 32; ++h)
                  if (r0 + r < rows && h * 32 + lane < cols) to[h * 32] = o[r][h];
                to += a.ldy;
              }
            }
          }
          __syncwarp();
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
      __syncwarp();
      if (lane == 0) {
        if constexpr (CG == 2) {
          asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];\n" ::"r"(map_to_rank(acc_empty_bar(buf), 0)) : "memory");
        } else {
          mbar_arrive(acc_empty_bar(buf));
        }
      }
    }
  }

  if constexpr (CG == 1 && SWAP && BN <= 64) {
    if (split > 1) {
      // Every CTA of the cluster finishes BN / split of the tile's tokens: the others send it their sums for them.
      __syncwarp();
      cluster_sync();   // all MMAs are done and all stages read: the rings may be written
      const int share_log2 = __ffs(BN / split) - 1, share = 1 << share_log2, row = (warp & 3) * 32 + lane;
      if (warp >= 4 && warp < 8) {
#pragma unroll
        for (int c = 0; c < BN; ++c) {
          const int to = c >> share_log2;
          const uint32_t at = smem0 + (uint32_t)(((int)rank * share + (c & (share - 1))) * 128 + row) * 4;
          asm volatile("st.shared::cluster.b32 [%0], %1;\n" ::"r"(map_to_rank(at, (uint32_t)to)), "r"(v[c]) : "memory");
        }
      }
      cluster_sync();
      if (warp >= 4 && warp < 8 && worker < tiles) {
        int ta, tb;
        place(worker, ta, tb);
        const int64_t o = (int64_t)ta * 128 + row;
        const float sa = o < a.rows_a ? __ldg(a.sa + o) : 0.f;
        for (int c = 0; c < share; ++c) {
          int sum = 0;
          for (int r = 0; r < split; ++r) {
            int part;
            asm volatile("ld.shared.b32 %0, [%1];\n" : "=r"(part) : "r"(smem0 + (uint32_t)((r * share + c) * 128 + row) * 4));
            sum += part;
          }
          const int64_t t = (int64_t)tb * BN + (int)rank * share + c;
          if (t < a.rows_b && o < a.rows_a) static_cast<T *>(a.y)[t * a.ldy + o] = from_f32<T>((float)sum * __ldg(a.sb + t) * sa);
        }
      }
    }
  }

  // No CTA gives its tensor memory back or leaves while another of the cluster may reach it or its shared memory.
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncwarp();
  cluster_sync();
  if (warp == 2) {
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    if constexpr (CG == 2)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(tmem_base), "r"(Cfg::kTmemCols) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem_base), "r"(Cfg::kTmemCols) : "memory");
  }
}

}  // namespace ssn
