// Query/key norm with rotary positions (include/agora_stage.h), forward and backward.
//
// A row is one head of one token: D values, one mean of squares, one pass.  Both directions move two (three) rows of D per
// row and compute a few operations per value, so HBM bounds them; what matters is wide loads, enough of them in flight and
// no second read.
//
// A row belongs to a group of G lanes (a power of two).  A lane's unit is V column PAIRS, so that no shuffle moves values:
// for halves one 16-byte piece at column i and one at i + rot_dim / 2, for adjacent pairs two pieces in a row.  The columns
// past rot_dim are paired in the same way (i with i + (D - rot_dim) / 2) and pass the rotation untouched.  A warp keeps the
// table row of its token in registers and goes through the token's heads, 32 / G at a time; blocks are dealt to the query
// and the key side by their numbers of heads, so that a warp needs one gain (and one gradient of it) only.
#include "stage_common.cuh"

#include <cmath>

namespace ssn {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kBlocksPerSm = 4;

struct RopeSide {
  const void *x, *dy;   // forward input; incoming gradient (backward)
  void *out;
  const void *w;        // gain or nullptr
  float *partial;       // [blocks x D] of this side, or nullptr (backward)
  int64_t x_token, x_head, dy_token, dy_head, out_token, out_head;
  int32_t heads, blocks;
  int32_t parts, passes;   // a token's heads are cut into `parts` of `passes` groups of rows
};

struct RopeArgs {
  RopeSide side[2];     // queries, keys
  const float *table;
  int64_t ldt;
  const int32_t *pos;
  int32_t *dev_status;
  int64_t n;
  int32_t d, rot, max_pos, seq_len, group_log2;
  float eps;
};

// Row of the table for token t, or -1
__device__ __forceinline__ int32_t table_row(const RopeArgs &a, int64_t t) {
  const int32_t p = a.pos != nullptr ? __ldg(a.pos + t)
                    : t <= 0x7fffffffLL ? (int32_t)((uint32_t)t % (uint32_t)a.seq_len) : (int32_t)(t % a.seq_len);
  if ((uint32_t)p < (uint32_t)a.max_pos) return p;
  if (a.dev_status != nullptr) atomicOr(a.dev_status, SSN_DEV_BAD_POS);
  return -1;
}

// The V pairs of a unit turned by the angle (sign = 1) or back (sign = -1).  lo and hi hold the unit's two pieces.
template <int V, bool ADJ>
__device__ __forceinline__ void turn(float (&lo)[V], float (&hi)[V], const float (&c)[V], const float (&s)[V], float sign) {
  if constexpr (!ADJ) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float a = lo[i], b = hi[i], ss = sign * s[i];
      lo[i] = a * c[i] - b * ss;
      hi[i] = b * c[i] + a * ss;
    }
  } else {
    float z[2 * V];
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] = lo[i], z[V + i] = hi[i];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float a = z[2 * i], b = z[2 * i + 1], ss = sign * s[i];
      z[2 * i] = a * c[i] - b * ss;
      z[2 * i + 1] = b * c[i] + a * ss;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) lo[i] = z[i], hi[i] = z[V + i];
  }
}

// NU units per lane (more than one only where V is small), BACK: the gradients, UB groups of rows in flight per warp
template <typename T, int V, int NU, bool ADJ, bool BACK, int UB>
__global__ void __launch_bounds__(kThreads, BACK ? 2 : kBlocksPerSm) qk_rope_kernel(const __grid_constant__ RopeArgs a) {
  __shared__ float sums[BACK ? kWarps : 1][BACK ? STAGE_MAX_HEAD_DIM : 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int side = (int)blockIdx.x >= a.side[0].blocks ? 1 : 0;
  const RopeSide &s = a.side[side];
  const int block = (int)blockIdx.x - (side ? a.side[0].blocks : 0);
  const int lg = a.group_log2, rows_per_pass = 32 >> lg, row = lane >> lg, unit0 = lane & ((1 << lg) - 1);
  const int half = a.rot >> 1, rest = (a.d - a.rot) >> 1;

  int lo_at[NU], hi_at[NU], pair[NU];
  bool mine[NU], turned[NU];
  Chunk<T, V> w_lo[NU], w_hi[NU];
  pdl_enter();
#pragma unroll
  for (int n = 0; n < NU; ++n) {
    pair[n] = (unit0 + (n << lg)) * V;
    mine[n] = 2 * pair[n] < a.d;
    turned[n] = pair[n] < half;
    if (ADJ) {
      lo_at[n] = 2 * pair[n];
      hi_at[n] = lo_at[n] + V;
    } else {
      lo_at[n] = turned[n] ? pair[n] : a.rot + pair[n] - half;
      hi_at[n] = lo_at[n] + (turned[n] ? half : rest);
    }
    if (mine[n] && s.w != nullptr) {
      w_lo[n].load(static_cast<const T *>(s.w) + lo_at[n]);
      w_hi[n].load(static_cast<const T *>(s.w) + hi_at[n]);
    } else {
      float one[V];
#pragma unroll
      for (int i = 0; i < V; ++i) one[i] = 1.f;
      w_lo[n].pack(one);
      w_hi[n].pack(one);
    }
  }
  float dw_lo[NU][V], dw_hi[NU][V];
  if (BACK) {
#pragma unroll
    for (int n = 0; n < NU; ++n)
#pragma unroll
      for (int i = 0; i < V; ++i) dw_lo[n][i] = dw_hi[n][i] = 0.f;
  }

  // this warp's part of the heads, and its tokens
  const int wid = block * kWarps + warp, slots = s.blocks * kWarps / s.parts;
  const int part = wid % s.parts;
  const float inv_d = 1.f / (float)a.d;
  for (int64_t t = wid / s.parts; wid < slots * s.parts && t < a.n; t += slots) {
    float c[NU][V], sn[NU][V];
    const int32_t p = a.rot > 0 ? table_row(a, t) : 0;
#pragma unroll
    for (int n = 0; n < NU; ++n) {
      if (mine[n] && turned[n] && p >= 0) {
        load_floats<V>(a.table + p * a.ldt + pair[n], c[n]);
        load_floats<V>(a.table + p * a.ldt + half + pair[n], sn[n]);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) c[n][i] = sn[n][i] = 0.f;
      }
    }
    const int first = part * s.passes * rows_per_pass;
    const int last = min(s.heads, first + s.passes * rows_per_pass);
    for (int h0 = first + row; h0 - row < last; h0 += UB * rows_per_pass) {
      Chunk<T, V> x_lo[UB][NU], x_hi[UB][NU], y_lo[BACK ? UB : 1][NU], y_hi[BACK ? UB : 1][NU];
#pragma unroll
      for (int b = 0; b < UB; ++b) {
        const int h = h0 + b * rows_per_pass;
        const T *x = static_cast<const T *>(s.x) + t * s.x_token + h * s.x_head;
        const T *dy = BACK ? static_cast<const T *>(s.dy) + t * s.dy_token + h * s.dy_head : nullptr;
#pragma unroll
        for (int n = 0; n < NU; ++n) {
          float zero[V];
#pragma unroll
          for (int i = 0; i < V; ++i) zero[i] = 0.f;
          if (mine[n] && h < last) {
            x_lo[b][n].load(x + lo_at[n]);
            x_hi[b][n].load(x + hi_at[n]);
            if (BACK) {
              y_lo[b][n].load(dy + lo_at[n]);
              y_hi[b][n].load(dy + hi_at[n]);
            }
          } else {
            x_lo[b][n].pack(zero);
            x_hi[b][n].pack(zero);
            if (BACK) {
              y_lo[b][n].pack(zero);
              y_hi[b][n].pack(zero);
            }
          }
        }
      }
#pragma unroll
      for (int b = 0; b < UB; ++b) {
        const int h = h0 + b * rows_per_pass;
        float sq = 0.f;
#pragma unroll
        for (int n = 0; n < NU; ++n)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            sq = fmaf(x_lo[b][n].get(i), x_lo[b][n].get(i), sq);
            sq = fmaf(x_hi[b][n].get(i), x_hi[b][n].get(i), sq);
          }
        for (int o = (1 << lg) >> 1; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
        const float r = __frsqrt_rn(fmaf(sq, inv_d, a.eps));
        T *out = static_cast<T *>(s.out) + t * s.out_token + h * s.out_head;
        if (!BACK) {
#pragma unroll
          for (int n = 0; n < NU; ++n) {
            float lo[V], hi[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
              lo[i] = x_lo[b][n].get(i) * r * w_lo[n].get(i);
              hi[i] = x_hi[b][n].get(i) * r * w_hi[n].get(i);
            }
            if (turned[n]) turn<V, ADJ>(lo, hi, c[n], sn[n], 1.f);
            if (mine[n] && h < last) {
              Chunk<T, V> o;
              o.pack(lo);
              o.store(out + lo_at[n]);
              o.pack(hi);
              o.store(out + hi_at[n]);
            }
          }
        } else {
          float g_lo[NU][V], g_hi[NU][V], inner = 0.f;
#pragma unroll
          for (int n = 0; n < NU; ++n) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
              g_lo[n][i] = y_lo[b][n].get(i);
              g_hi[n][i] = y_hi[b][n].get(i);
            }
            if (turned[n]) turn<V, ADJ>(g_lo[n], g_hi[n], c[n], sn[n], -1.f);
#pragma unroll
            for (int i = 0; i < V; ++i) {
              const float u_lo = x_lo[b][n].get(i) * r, u_hi = x_hi[b][n].get(i) * r;
              // a row past the last head, or a column past D, is made of zeros: it adds nothing
              dw_lo[n][i] = fmaf(g_lo[n][i], u_lo, dw_lo[n][i]);
              dw_hi[n][i] = fmaf(g_hi[n][i], u_hi, dw_hi[n][i]);
              g_lo[n][i] *= w_lo[n].get(i);
              g_hi[n][i] *= w_hi[n].get(i);
              inner = fmaf(g_lo[n][i], u_lo, inner);
              inner = fmaf(g_hi[n][i], u_hi, inner);
            }
          }
          for (int o = (1 << lg) >> 1; o > 0; o >>= 1) inner += __shfl_xor_sync(0xffffffffu, inner, o);
          inner *= inv_d;
#pragma unroll
          for (int n = 0; n < NU; ++n) {
            float lo[V], hi[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
              lo[i] = r * fmaf(-(x_lo[b][n].get(i) * r), inner, g_lo[n][i]);
              hi[i] = r * fmaf(-(x_hi[b][n].get(i) * r), inner, g_hi[n][i]);
            }
            if (mine[n] && h < last) {
              Chunk<T, V> o;
              o.pack(lo);
              o.store(out + lo_at[n]);
              o.pack(hi);
              o.store(out + hi_at[n]);
            }
          }
        }
      }
    }
  }

  if (BACK && s.partial != nullptr) {   // the block's share of dw: lanes of one column, then warps, always in the same order
#pragma unroll
    for (int n = 0; n < NU; ++n)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        for (int o = 16; o >= (1 << lg); o >>= 1) {
          dw_lo[n][i] += __shfl_xor_sync(0xffffffffu, dw_lo[n][i], o);
          dw_hi[n][i] += __shfl_xor_sync(0xffffffffu, dw_hi[n][i], o);
        }
        if (row == 0 && mine[n]) {
          sums[warp][lo_at[n] + i] = dw_lo[n][i];
          sums[warp][hi_at[n] + i] = dw_hi[n][i];
        }
      }
    __syncthreads();
    for (int col = threadIdx.x; col < a.d; col += kThreads) {
      float total = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) total += sums[w][col];
      s.partial[(int64_t)block * a.d + col] = total;
    }
  }
}

// dw[col] = sum over the blocks' partial sums, in 64 bits.  A block takes 32 columns of one side.
struct GainArgs {
  const float *partial[2];
  float *dw[2];
  int32_t blocks[2], d;
};
__global__ void __launch_bounds__(1024) qk_rope_gain_kernel(const GainArgs a) {
  __shared__ double sums[32][33];
  const int side = blockIdx.y, col = blockIdx.x * 32 + threadIdx.x;
  pdl_enter();
  double total = 0.0;
  if (col < a.d && a.dw[side] != nullptr)
    for (int b = threadIdx.y; b < a.blocks[side]; b += 32) total += (double)a.partial[side][(int64_t)b * a.d + col];
  sums[threadIdx.y][threadIdx.x] = total;
  __syncthreads();
  if (threadIdx.y == 0 && col < a.d && a.dw[side] != nullptr) {
    for (int y = 1; y < 32; ++y) total += sums[y][threadIdx.x];
    a.dw[side][col] = (float)total;
  }
}

// One angle per thread; sincos in 64 bits is what bounds it, and it runs once per model.
__global__ void __launch_bounds__(256) rope_table_kernel(float *table, int64_t ldt, int32_t max_pos, int32_t rot, double log_theta) {
  pdl_enter();
  const int half = rot >> 1;
  const int64_t total = (int64_t)max_pos * half, stride = (int64_t)gridDim.x * blockDim.x;
  for (int64_t e = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; e < total; e += stride) {
    const int64_t p = e / half;
    const int i = (int)(e - p * half);
    double sn, cs;
    sincos((double)p * exp(-log_theta * (2.0 * i / rot)), &sn, &cs);
    table[p * ldt + i] = (float)cs;
    table[p * ldt + half + i] = (float)sn;
  }
}

ssn_status_t check_op(const stage_qk_rope_t *op) {
  if (op == nullptr) return SSN_ERR_NULL;
  if (op->dtype != SSN_F32 && op->dtype != SSN_BF16) return SSN_ERR_DTYPE;
  if (op->pairing != STAGE_PAIR_HALVES && op->pairing != STAGE_PAIR_ADJACENT) return SSN_ERR_DTYPE;
  if (op->head_dim < 2 || op->head_dim > STAGE_MAX_HEAD_DIM || (op->head_dim & 1)) return SSN_ERR_SHAPE;
  if (op->rot_dim < 0 || op->rot_dim > op->head_dim || (op->rot_dim & 1)) return SSN_ERR_SHAPE;
  if (!(op->eps >= 0.f) || std::isinf(op->eps)) return SSN_ERR_SHAPE;
  if (op->rot_dim > 0) {
    if (op->table == nullptr) return SSN_ERR_NULL;
    if (op->ldt < op->rot_dim || op->max_pos < 1) return SSN_ERR_SHAPE;
  }
  return SSN_OK;
}

// A [n x heads x D] tensor: strides that cannot leave 63 bits, and for an output rows that keep apart
ssn_status_t check_heads(const void *x, int64_t token, int64_t head, int64_t n, int32_t heads, int32_t d, size_t item, bool output) {
  if (heads == 0) return SSN_OK;
  constexpr int64_t kFar = (int64_t)1 << 60;
  if (token < 0 || head < 0 || heads > 65536) return SSN_ERR_SHAPE;
  if ((heads > 1 && head > kFar / (heads - 1)) || (n > 1 && token > kFar / (n - 1))) return SSN_ERR_SHAPE;
  if (output) {
    if (heads > 1 && head < d) return SSN_ERR_SHAPE;
    if (n > 1 && token < d) return SSN_ERR_SHAPE;
    if (heads > 1 && n > 1 && token < (heads - 1) * head + d && head < (n - 1) * token + d) return SSN_ERR_SHAPE;
  }
  if (x == nullptr) return SSN_ERR_NULL;
  return aligned_to(x, item) ? SSN_OK : SSN_ERR_SHAPE;
}

// Elements per piece (a power of two, 16 bytes at most) that every address and stride allows
struct Width {
  int v;
  explicit Width(size_t item) : v((int)(16 / item)) {}
  void address(const void *p, size_t item) {
    while (v > 1 && (reinterpret_cast<uintptr_t>(p) % (v * item)) != 0) v >>= 1;
  }
  void stride(int64_t s) {
    while (v > 1 && s % v != 0) v >>= 1;
  }
  void table(const void *p, int64_t ld) {
    while (v > 1 && (reinterpret_cast<uintptr_t>(p) % (4 * (v < 4 ? v : 4)) != 0 || ld % (v < 4 ? v : 4) != 0)) v >>= 1;
  }
};

void plan_side(RopeSide &s, int64_t n, int rows_per_pass, int max_blocks) {
  s.parts = s.passes = 1;
  s.blocks = 0;
  if (s.heads == 0 || n == 0) return;
  // A warp goes through all heads of a token when there are tokens enough for every warp; few tokens are cut into parts.
  const int64_t warps = (int64_t)max_blocks * kWarps, passes = (s.heads + rows_per_pass - 1) / rows_per_pass;
  int64_t each = n * passes / warps;
  each = each < 1 ? 1 : (each > passes ? passes : each);
  s.passes = (int32_t)each;
  s.parts = (int32_t)((passes + each - 1) / each);
  const int64_t need = (n * s.parts + kWarps - 1) / kWarps, least = (s.parts + kWarps - 1) / kWarps;
  s.blocks = (int32_t)(need < max_blocks ? need : max_blocks);
  if (s.blocks < least) s.blocks = (int32_t)least;   // a slot for every part
}

// The most blocks a side gets: the resident ones, dealt by heads
int side_blocks(int sms, int per_sm, int32_t heads, int32_t other) {
  if (heads == 0) return 0;
  const int64_t b = (int64_t)sms * per_sm * heads / ((int64_t)heads + other);
  return b < 1 ? 1 : (int)b;
}

template <typename T, bool ADJ, bool BACK>
cudaError_t launch_width(const RopeArgs &a, int v, cudaStream_t stream) {
  const unsigned grid = (unsigned)(a.side[0].blocks + a.side[1].blocks);
  if constexpr (sizeof(T) == 2) {
    if (v == 8) return launch_dependent(qk_rope_kernel<T, 8, 1, ADJ, BACK, 2>, grid, kThreads, 0, stream, 1, a);
  }
  if (v >= 4) return launch_dependent(qk_rope_kernel<T, 4, 1, ADJ, BACK, 2>, grid, kThreads, 0, stream, 1, a);
  if (v == 2) return launch_dependent(qk_rope_kernel<T, 2, 2, ADJ, BACK, 1>, grid, kThreads, 0, stream, 1, a);
  return launch_dependent(qk_rope_kernel<T, 1, 4, ADJ, BACK, 1>, grid, kThreads, 0, stream, 1, a);
}

template <bool BACK>
ssn_status_t launch_rope(const stage_qk_rope_t *op, RopeArgs &a, int v, cudaStream_t stream) {
  const bool adj = op->pairing == STAGE_PAIR_ADJACENT;
  cudaError_t e;
  if (op->dtype == SSN_F32)
    e = adj ? launch_width<float, true, BACK>(a, v, stream) : launch_width<float, false, BACK>(a, v, stream);
  else
    e = adj ? launch_width<__nv_bfloat16, true, BACK>(a, v, stream) : launch_width<__nv_bfloat16, false, BACK>(a, v, stream);
  return launched(e);
}

// Lanes per row and the blocks of both sides
void plan(const stage_qk_rope_t *op, RopeArgs &a, int v, int per_sm) {
  const int units = (op->head_dim / 2 + v - 1) / v;
  a.group_log2 = 0;
  while ((1 << a.group_log2) < units && a.group_log2 < 5) ++a.group_log2;
  const int sms = stage_sm_count(), rows = 32 >> a.group_log2;
  for (int i = 0; i < 2; ++i) plan_side(a.side[i], a.n, rows, side_blocks(sms, per_sm, a.side[i].heads, a.side[1 - i].heads));
}

void fill(const stage_qk_rope_t *op, RopeArgs &a, const int32_t *pos, int64_t n, int32_t seq_len) {
  a.table = op->table;
  a.ldt = op->ldt;
  a.pos = pos;
  a.dev_status = op->dev_status;
  a.n = n;
  a.d = op->head_dim;
  a.rot = op->rot_dim;
  a.max_pos = op->max_pos;
  a.seq_len = seq_len;
  a.eps = op->eps;
  a.side[0].w = op->wq;
  a.side[1].w = op->wk;
}

int width_of(const stage_qk_rope_t *op, const RopeArgs &a, bool back) {
  const size_t item = op->dtype == SSN_F32 ? 4 : 2;
  Width w(item);
  w.stride(a.rot / 2);
  w.stride((a.d - a.rot) / 2);
  if (a.rot > 0) w.table(a.table, a.ldt);
  for (const RopeSide &s : a.side) {
    if (s.heads == 0) continue;
    w.address(s.x, item);
    w.address(s.out, item);
    if (s.w != nullptr) w.address(s.w, item);
    for (int64_t st : {s.x_token, s.x_head, s.out_token, s.out_head}) w.stride(st);
    if (back) {
      w.address(s.dy, item);
      w.stride(s.dy_token);
      w.stride(s.dy_head);
    }
  }
  return w.v;
}

constexpr int kBackPerSm = 2;   // resident blocks of the backward kernel (its launch bounds)

}  // namespace
}  // namespace ssn

using namespace ssn;

extern "C" {

ssn_status_t stage_rope_table(float *table, int64_t ldt, int32_t max_pos, int32_t rot_dim, double theta, void *stream) {
  if (rot_dim < 2 || (rot_dim & 1) || max_pos < 0 || ldt < rot_dim || !(theta > 0.0) || std::isinf(theta)) return SSN_ERR_SHAPE;
  if (max_pos == 0) return SSN_OK;
  if (table == nullptr) return SSN_ERR_NULL;
  const int64_t blocks = ((int64_t)max_pos * (rot_dim / 2) + 255) / 256, cap = (int64_t)stage_sm_count() * 8;
  return launched(launch_dependent(rope_table_kernel, (unsigned)(blocks < cap ? blocks : cap), 256, 0, static_cast<cudaStream_t>(stream), 1,
                                   table, ldt, max_pos, rot_dim, std::log(theta)));
}

ssn_status_t stage_qk_rope_forward(const stage_qk_rope_t *op, const void *q, int64_t q_token, int64_t q_head, int32_t q_heads,
                                   const void *k, int64_t k_token, int64_t k_head, int32_t k_heads, void *q_out,
                                   int64_t qo_token, int64_t qo_head, void *k_out, int64_t ko_token, int64_t ko_head,
                                   const int32_t *pos, int64_t n_tokens, int32_t seq_len, void *stream) {
  ssn_status_t st = check_op(op);
  if (st != SSN_OK) return st;
  if (n_tokens < 0 || n_tokens > (int64_t)1 << 40 || q_heads < 0 || k_heads < 0) return SSN_ERR_SHAPE;
  if (n_tokens == 0 || (q_heads == 0 && k_heads == 0)) return SSN_OK;
  if (op->rot_dim > 0 && pos == nullptr && seq_len < 1) return SSN_ERR_SHAPE;
  const int32_t d = op->head_dim;
  const size_t item = op->dtype == SSN_F32 ? 4 : 2;
  if ((st = check_heads(q, q_token, q_head, n_tokens, q_heads, d, item, false)) != SSN_OK) return st;
  if ((st = check_heads(k, k_token, k_head, n_tokens, k_heads, d, item, false)) != SSN_OK) return st;
  if ((st = check_heads(q_out, qo_token, qo_head, n_tokens, q_heads, d, item, true)) != SSN_OK) return st;
  if ((st = check_heads(k_out, ko_token, ko_head, n_tokens, k_heads, d, item, true)) != SSN_OK) return st;
  RopeArgs a{};
  fill(op, a, pos, n_tokens, seq_len);
  const RopeSide qs{q, nullptr, q_out, op->wq, nullptr, q_token, q_head, 0, 0, qo_token, qo_head, q_heads, 0, 1, 1};
  const RopeSide ks{k, nullptr, k_out, op->wk, nullptr, k_token, k_head, 0, 0, ko_token, ko_head, k_heads, 0, 1, 1};
  a.side[0] = qs;
  a.side[1] = ks;
  const int v = width_of(op, a, false);
  plan(op, a, v, kBlocksPerSm);
  return launch_rope<false>(op, a, v, static_cast<cudaStream_t>(stream));
}

// Partial sums of at most the resident blocks, D floats each (a side never has fewer than a slot per part of its heads)
size_t stage_qk_rope_workspace_bytes(const stage_qk_rope_t *op, int64_t n_tokens, int32_t q_heads, int32_t k_heads) {
  if (check_op(op) != SSN_OK || n_tokens <= 0 || q_heads < 0 || k_heads < 0) return 0;
  const int64_t resident = (int64_t)stage_sm_count() * kBackPerSm + 2;
  return (size_t)(resident + ((int64_t)q_heads + k_heads) / kWarps + 2) * op->head_dim * sizeof(float);
}

ssn_status_t stage_qk_rope_backward(const stage_qk_rope_t *op, const void *dq, int64_t dq_token, int64_t dq_head,
                                    const void *dk, int64_t dk_token, int64_t dk_head, const void *q, int64_t q_token,
                                    int64_t q_head, int32_t q_heads, const void *k, int64_t k_token, int64_t k_head,
                                    int32_t k_heads, void *dq_in, int64_t dqi_token, int64_t dqi_head, void *dk_in,
                                    int64_t dki_token, int64_t dki_head, float *dwq, float *dwk, const int32_t *pos,
                                    int64_t n_tokens, int32_t seq_len, void *workspace, size_t workspace_bytes, void *stream) {
  ssn_status_t st = check_op(op);
  if (st != SSN_OK) return st;
  if (n_tokens < 0 || n_tokens > (int64_t)1 << 40 || q_heads < 0 || k_heads < 0) return SSN_ERR_SHAPE;
  const bool rows = n_tokens > 0 && (q_heads > 0 || k_heads > 0);
  const int32_t d = op->head_dim;
  const size_t item = op->dtype == SSN_F32 ? 4 : 2;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  RopeArgs a{};
  int launches = 0;
  if (rows) {
    if (op->rot_dim > 0 && pos == nullptr && seq_len < 1) return SSN_ERR_SHAPE;
    if ((st = check_heads(dq, dq_token, dq_head, n_tokens, q_heads, d, item, false)) != SSN_OK) return st;
    if ((st = check_heads(dk, dk_token, dk_head, n_tokens, k_heads, d, item, false)) != SSN_OK) return st;
    if ((st = check_heads(q, q_token, q_head, n_tokens, q_heads, d, item, false)) != SSN_OK) return st;
    if ((st = check_heads(k, k_token, k_head, n_tokens, k_heads, d, item, false)) != SSN_OK) return st;
    if ((st = check_heads(dq_in, dqi_token, dqi_head, n_tokens, q_heads, d, item, true)) != SSN_OK) return st;
    if ((st = check_heads(dk_in, dki_token, dki_head, n_tokens, k_heads, d, item, true)) != SSN_OK) return st;
    if ((dwq != nullptr || dwk != nullptr) &&
        (workspace == nullptr || !aligned_to(workspace, 16) || workspace_bytes < stage_qk_rope_workspace_bytes(op, n_tokens, q_heads, k_heads)))
      return SSN_ERR_WORKSPACE;
    fill(op, a, pos, n_tokens, seq_len);
    const RopeSide qs{q, dq, dq_in, op->wq, nullptr, q_token, q_head, dq_token, dq_head, dqi_token, dqi_head, q_heads, 0, 1, 1};
    const RopeSide ks{k, dk, dk_in, op->wk, nullptr, k_token, k_head, dk_token, dk_head, dki_token, dki_head, k_heads, 0, 1, 1};
    a.side[0] = qs;
    a.side[1] = ks;
    const int v = width_of(op, a, true);
    plan(op, a, v, kBackPerSm);
    float *partial = static_cast<float *>(workspace);
    if (dwq != nullptr) a.side[0].partial = partial;
    if (dwk != nullptr) a.side[1].partial = partial + (int64_t)a.side[0].blocks * d;
    if ((st = launch_rope<true>(op, a, v, s)) != SSN_OK) return st;
    ++launches;
  }
  if (dwq != nullptr || dwk != nullptr) {
    GainArgs g{{a.side[0].partial, a.side[1].partial}, {dwq, dwk}, {a.side[0].blocks, a.side[1].blocks}, d};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((d + 31) / 32), 2);
    cfg.blockDim = dim3(32, 32);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
    cfg.numAttrs = cudaStreamIsCapturing(s, &capturing) == cudaSuccess && capturing == cudaStreamCaptureStatusNone ? 1 : 0;
    return launched(cudaLaunchKernelEx(&cfg, qk_rope_gain_kernel, g));
  }
  return SSN_OK;
}

}  // extern "C"
