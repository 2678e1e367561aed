// Dispatch of the tcgen05 8-bit product (see stage_int8_umma.cuh).
#include "stage_int8_umma.cuh"

#include <algorithm>

#include "codec_tensor_maps.h"

namespace ssn {
namespace {

template <int CG, int BN, bool SWAP, typename T, bool RAGGED = false>
cudaError_t launch_tiles(const Int8Matmul &m, int split, int sm_count, cudaStream_t stream) {
  using Cfg = Int8Config<CG, BN, SWAP, RAGGED>;
  static std::atomic<uint64_t> allowed{0};
  auto kernel = int8_umma_kernel<CG, BN, SWAP, RAGGED, T>;
  Int8Maps maps{};
  Int8Args a{};
  a.a = SWAP ? m.wq : m.xq;
  a.b = SWAP ? m.xq : m.wq;
  const int64_t ra = SWAP ? m.outer : m.n, rb = SWAP ? m.n : m.outer;
  a.lda = SWAP ? m.ldw : m.ldx;
  a.ldb = SWAP ? m.ldx : m.ldw;
  a.inner = (int32_t)m.inner;
  if (!RAGGED && (!make_sw128_map_u8(&maps.a, a.a, ra, m.inner, a.lda, 128) || !make_sw128_map_u8(&maps.b, a.b, rb, m.inner, a.ldb, Cfg::kBRows)))
    return cudaErrorNotSupported;
  a.sa = SWAP ? m.ws : m.xs;
  a.sb = SWAP ? m.xs : m.ws;
  a.y = m.y;
  a.ldy = m.ldy;
  a.rows_a = (int32_t)ra;
  a.rows_b = (int32_t)rb;
  a.steps = (int32_t)((m.inner + kInt8Step - 1) / kInt8Step);
  a.tiles_a = (int32_t)((ra + 128 * CG - 1) / (128 * CG));
  a.tiles_b = (int32_t)((rb + BN - 1) / BN);
  a.dev_status = m.dev_status;
  note_kernel(STAGE_KERNEL_INT8_UMMA, BN | (CG == 2 ? STAGE_KVAR_PAIR : 0) | (SWAP ? STAGE_KVAR_SWAP : 0) | (split > 1 ? STAGE_KVAR_SPLIT : 0) |
                                          (RAGGED ? STAGE_KVAR_ANYWHERE : 0));
  cudaError_t e = allow_dynamic_smem(kernel, Cfg::kSmemBytes, allowed);
  if (e != cudaSuccess) return e;
  const int cluster = CG == 2 ? 2 : split;
  const int64_t tiles = (int64_t)a.tiles_a * a.tiles_b;
  int64_t workers = split > 1 ? tiles : sm_count / CG;   // a splitting cluster has one tile
  if (workers > tiles) workers = tiles;
  return launch_dependent(kernel, (unsigned)(workers * cluster), Cfg::kThreads, Cfg::kSmemBytes, stream, cluster, a, maps);
}

// CTAs per tile of 128 channels x bn tokens, while there are SMs for them and each keeps a few steps of the inner dimension.  Not
// every SM of a GPC is in a cluster: a sixteenth cluster of eight would run after the others (100 x 4096 x 1024: 17.8 us).
int split_of(const Int8Matmul &m, int bn, int sms) {
  const int64_t steps = (m.inner + kInt8Step - 1) / kInt8Step, tiles = (m.outer + 127) / 128 * ((m.n + bn - 1) / bn);
  int split = 1;
  while (split < 8 && tiles * split * 2 <= (split == 4 ? sms * 13 / 16 : sms * 7 / 8) && steps >= split * 4) split *= 2;
  return split;
}

template <typename T> cudaError_t launch_ragged(const Int8Matmul &m, int sms, cudaStream_t stream) {
  if (m.n <= 16) return launch_tiles<1, 16, true, T, true>(m, split_of(m, 16, sms), sms, stream);
  const int split = split_of(m, 64, sms);   // few tiles: several CTAs for each
  if (m.n <= 64 || split > 1) return launch_tiles<1, 64, true, T, true>(m, split, sms, stream);
  return launch_tiles<1, 128, false, T, true>(m, 1, sms, stream);
}

template <typename T> cudaError_t launch_typed(const Int8Matmul &m, int sms, cudaStream_t stream) {
  if (m.n <= 16) return launch_tiles<1, 16, true, T>(m, split_of(m, 16, sms), sms, stream);
  if (m.n <= 32) return launch_tiles<1, 32, true, T>(m, split_of(m, 32, sms), sms, stream);
  if (m.n <= 64) return launch_tiles<1, 64, true, T>(m, split_of(m, 64, sms), sms, stream);
  // The shape whose waves of tiles take the least time: a step of a wave of pairs of 256 x 256 takes about 0.38 us, of CTAs of
  // 128 x 256 0.42 (each loads B for itself), of CTAs of 128 x 128 0.28; the output of a tile takes 4.0, 3.5 and 3.0 us, which
  // is also the least time of a wave, and is hidden behind the next wave but for the last one.  Measured (us; pairs, CTAs of 256,
  // CTAs of 128): 777 x 2000 x 5003 21.8 / 16.4 / 19.1, 128 x 4096 x 4096 15.2 / 14.5 / 13.2, 256 x 4096 x 128256 109 / 128 / 150,
  // 16384 x 256 x 4096 59 / 52 / 60.
  const double steps = (double)((m.inner + kInt8Step - 1) / kInt8Step);
  auto time = [&](int64_t ta, int64_t bn, int64_t workers, double step, double rest) {
    const int64_t tiles = ta * ((m.outer + bn - 1) / bn), waves = (tiles + workers - 1) / workers;
    return (double)waves * (step * steps > rest ? step * steps : rest) + rest;
  };
  const int64_t half = (m.n + 127) / 128, whole = (m.n + 255) / 256;
  const double pairs = time(whole, 256, sms / 2, 0.38, 4.0), wide = time(half, 256, sms, 0.42, 3.5), narrow = time(half, 128, sms, 0.28, 3.0);
  const int split = split_of(m, 64, sms);   // few tiles: several CTAs for each
  if (split > 1 && steps / split * 0.2 + 7.0 < std::min(pairs, std::min(wide, narrow))) return launch_tiles<1, 64, true, T>(m, split, sms, stream);
  if (wide < pairs && wide <= narrow) return launch_tiles<1, 256, false, T>(m, 1, sms, stream);
  if (narrow < pairs) return launch_tiles<1, 128, false, T>(m, 1, sms, stream);
  return launch_tiles<2, 256, false, T>(m, 1, sms, stream);
}

}  // namespace

cudaError_t launch_int8_umma(const Int8Matmul &m, bool f32, bool rows16, int sm_count, cudaStream_t stream) {
  if (sm_count < 2) sm_count = 2;
  constexpr int64_t kPitch = (int64_t)1 << 40;   // of a tensor map
  if (rows16 && m.ldx < kPitch && m.ldw < kPitch) {
    const cudaError_t e = f32 ? launch_typed<float>(m, sm_count, stream) : launch_typed<__nv_bfloat16>(m, sm_count, stream);
    if (e != cudaErrorNotSupported) return e;
  }
  return f32 ? launch_ragged<float>(m, sm_count, stream) : launch_ragged<__nv_bfloat16>(m, sm_count, stream);
}

}  // namespace ssn
