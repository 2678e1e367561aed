// Dispatch of the tcgen05 8-bit product (see stage_int8_umma.cuh).
#include "stage_int8_umma.cuh"

#include "codec_tensor_maps.h"

namespace ssn {
namespace {

template <int CG, int BN, bool SWAP, typename T>
cudaError_t launch_tiles(const Int8Matmul &m, int split, int sm_count, cudaStream_t stream) {
  using Cfg = Int8Config<CG, BN, SWAP>;
  static std::atomic<uint64_t> allowed{0};
  auto kernel = int8_umma_kernel<CG, BN, SWAP, T>;
  Int8Maps maps;
  const int8_t *pa = SWAP ? m.wq : m.xq, *pb = SWAP ? m.xq : m.wq;
  const int64_t ra = SWAP ? m.outer : m.n, rb = SWAP ? m.n : m.outer, la = SWAP ? m.ldw : m.ldx, lb = SWAP ? m.ldx : m.ldw;
  if (!make_sw128_map_u8(&maps.a, pa, ra, m.inner, la, 128) || !make_sw128_map_u8(&maps.b, pb, rb, m.inner, lb, Cfg::kBRows))
    return cudaErrorNotSupported;
  Int8Args a{};
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
  cudaError_t e = allow_dynamic_smem(kernel, Cfg::kSmemBytes, allowed);
  if (e != cudaSuccess) return e;
  const int cluster = CG == 2 ? 2 : split;
  const int64_t tiles = (int64_t)a.tiles_a * a.tiles_b;
  int64_t workers = split > 1 ? tiles : sm_count / CG;   // a splitting cluster has one tile
  if (workers > tiles) workers = tiles;
  return launch_dependent(kernel, (unsigned)(workers * cluster), kInt8Threads, Cfg::kSmemBytes, stream, cluster, a, maps);
}

template <typename T> cudaError_t launch_typed(const Int8Matmul &m, int sms, cudaStream_t stream) {
  const int64_t steps = (m.inner + kInt8Step - 1) / kInt8Step;
  if (m.n <= 256) {   // few tokens: weights on the M side
    const int64_t tiles = (m.outer + 127) / 128;
    int split = 1;   // CTAs per tile, while there are SMs for them and each keeps a few steps
    while (m.n <= 64 && split < 8 && tiles * split * 2 <= sms && steps >= split * 4) split *= 2;
    if (m.n <= 16) return launch_tiles<1, 16, true, T>(m, split, sms, stream);
    if (m.n <= 32) return launch_tiles<1, 32, true, T>(m, split, sms, stream);
    if (m.n <= 64) return launch_tiles<1, 64, true, T>(m, split, sms, stream);
    if (m.n <= 128) return launch_tiles<1, 128, true, T>(m, 1, sms, stream);
    return launch_tiles<1, 256, true, T>(m, 1, sms, stream);
  }
  // The tile width whose last wave leaves the fewest SMs idle, a narrower tile counted as slower per column.
  const int64_t pairs = sms / 2 > 0 ? sms / 2 : 1, ta = (m.n + 255) / 256;
  auto cost = [&](int64_t bn, int64_t per_tile) { return (ta * ((m.outer + bn - 1) / bn) + pairs - 1) / pairs * per_tile; };
  if (cost(128, 150) < cost(256, 256)) return launch_tiles<2, 128, false, T>(m, 1, sms, stream);
  return launch_tiles<2, 256, false, T>(m, 1, sms, stream);
}

}  // namespace

cudaError_t launch_int8_umma(const Int8Matmul &given, bool f32, int sm_count, cudaStream_t stream) {
  Int8Matmul m = given;   // the pitch of a single row does not matter
  if (m.n == 1) m.ldx = (m.inner + 15) / 16 * 16;
  if (m.outer == 1) m.ldw = (m.inner + 15) / 16 * 16;
  if (((reinterpret_cast<uintptr_t>(m.xq) | reinterpret_cast<uintptr_t>(m.wq) | (uintptr_t)m.ldx | (uintptr_t)m.ldw) & 15) != 0)
    return cudaErrorNotSupported;
  // row coordinates and strides a tensor map can hold
  constexpr int64_t kRows = 0x7fffff00, kPitch = (int64_t)1 << 40;
  if (m.n > kRows || m.outer > kRows || m.ldx >= kPitch || m.ldw >= kPitch || sm_count < 2) return cudaErrorNotSupported;
  return f32 ? launch_typed<float>(m, sm_count, stream) : launch_typed<__nv_bfloat16>(m, sm_count, stream);
}

}  // namespace ssn
