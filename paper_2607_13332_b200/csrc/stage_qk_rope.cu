// Query/key norm with rotary positions (include/agora_stage.h), forward and backward.
//
// A row is one head of one token: D values, one mean of squares, one pass.  Both directions move two (three) rows of D per
// row and compute a few operations per value: HBM bounds the forward pass (65536 tokens x 40 heads of 128 bf16 in 217 us,
// 6.2 TB/s, 0.95 of a copy), HBM and instruction issue the gradients (32768 tokens in 179 us, 5.6 TB/s, 0.86).
//
// A row belongs to a group of G lanes (a power of two).  A lane's unit is V column PAIRS, so that no shuffle moves values:
// for halves one 16-byte piece at column i and one at i + rot_dim / 2, for adjacent pairs at i and i + D / 2.  The halves'
// columns past rot_dim are paired in the same way (i with i + (D - rot_dim) / 2) and pass the rotation untouched.  A warp keeps the
// table row of its token in registers and goes through the token's heads, 32 / G at a time; blocks are dealt to the query
// and the key side by their numbers of heads, so that a warp needs one gain (and one gradient of it) only.  Rows are loaded
// through a ring in shared memory: loads into registers, as many as fit, left the forward pass at 259 us.
#include "stage_common.cuh"

#include <cmath>

namespace ssn {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
// Resident blocks, and passes of rows on their way per warp.  65536 x 40 heads of 128 bf16 forward: two blocks three passes ahead
// 217 us, two 234, four or six 248, three blocks spill (336).  The gradients of 32768: two passes ahead 183 us, three or four 179.
constexpr int kPerSm = 2;
constexpr int kForwardAhead = 3, kBackAhead = 3;

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
  int32_t table_bytes, wide_table;   // a table row's room in shared memory; its rows are on 16-byte boundaries
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

// V column pairs (a, b) in two pieces of V elements: the halves' pieces are the a and the b; of adjacent pairs either piece holds
// V / 2, or its half of the only one
template <typename T, int V, bool ADJ> struct Unit {
  Chunk<T, V> p0, p1;
  static __device__ __forceinline__ int a_column(int at0, int at1, int i) { return !ADJ || V == 1 ? at0 + i : 2 * i < V ? at0 + 2 * i : at1 + 2 * i - V; }
  static __device__ __forceinline__ int b_column(int at0, int at1, int i) { return !ADJ || V == 1 ? at1 + i : a_column(at0, at1, i) + 1; }
  __device__ __forceinline__ void load(const T *x, int at0, int at1) {
    p0.load(x + at0);
    p1.load(x + at1);
  }
  __device__ __forceinline__ void store(T *x, int at0, int at1) const {
    p0.store(x + at0);
    p1.store(x + at1);
  }
  // from this lane's place in a ring: the 32 lanes' first pieces, then their second ones
  __device__ __forceinline__ void take(const unsigned char *place) {
    p0.load(reinterpret_cast<const T *>(place));
    p1.load(reinterpret_cast<const T *>(place + 32 * V * sizeof(T)));
  }
  __device__ __forceinline__ void get(float (&a)[V], float (&b)[V]) const {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      a[i] = !ADJ ? p0.get(i) : 2 * i < V ? p0.get(2 * i < V ? 2 * i : 0) : p1.get(2 * i < V ? 0 : 2 * i - V);
      b[i] = !ADJ ? p1.get(i) : 2 * i + 1 < V ? p0.get(2 * i + 1 < V ? 2 * i + 1 : 0) : p1.get(2 * i + 1 < V ? 0 : 2 * i + 1 - V);
    }
  }
  __device__ __forceinline__ void pack(const float (&a)[V], const float (&b)[V]) {
    if constexpr (!ADJ) {
      p0.pack(a);
      p1.pack(b);
    } else {
      float z0[V], z1[V];
#pragma unroll
      for (int i = 0; i < 2 * V; ++i) (i < V ? z0[i < V ? i : 0] : z1[i < V ? 0 : i - V]) = i & 1 ? b[i >> 1] : a[i >> 1];
      p0.pack(z0);
      p1.pack(z1);
    }
  }
};

// Copies a piece to shared memory behind this thread's back; two bytes are more than cp.async can (they wait here)
template <int BYTES> __device__ __forceinline__ void copy_piece(unsigned char *to, const void *from) {
  const uint32_t at = smem_address(to);
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(at), "l"(from) : "memory");
  else if constexpr (BYTES >= 4) asm volatile("cp.async.ca.shared.global [%0], [%1], %2;\n" ::"r"(at), "l"(from), "n"(BYTES) : "memory");
  else *reinterpret_cast<uint16_t *>(to) = *static_cast<const uint16_t *>(from);
}
template <int BYTES> __device__ __forceinline__ void clear_piece(unsigned char *to) {
  RawBytes<BYTES> zero = {};
  *reinterpret_cast<RawBytes<BYTES> *>(to) = zero;
}

__device__ __forceinline__ float group_sum(float x, int group_log2) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1)
    if (o < (1 << group_log2)) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// How pairs of columns come together: both in a lane's unit (HALVES, ADJACENT), or, for halves whose distance is no multiple of V,
// from the row in shared memory (CROSSED): a lane turns the columns of its two pieces and reads their partners one by one.
enum Pairs { HALVES, ADJACENT, CROSSED };

// NU units per lane (more than one only where V is small).  A warp's rows come through a ring in shared memory: every lane
// copies its own pieces kAhead passes ahead (cp.async, no registers held), and the warp together the table rows of the tokens
// that these passes begin.
template <typename T, int V, int NU, Pairs PAIRS, bool BACK, bool FULL>
__global__ void __launch_bounds__(kThreads, kPerSm) qk_rope_kernel(const __grid_constant__ RopeArgs a) {
  constexpr int P = BACK ? kBackAhead : kForwardAhead, kPieceBytes = V * (int)sizeof(T), kUnitBytes = 2 * 32 * kPieceBytes;
  constexpr int kPassBytes = (BACK ? 2 : 1) * NU * kUnitBytes, kTables = P + 1;
  extern __shared__ __align__(16) unsigned char dyn[];
  __shared__ float sums[BACK ? kWarps : 1][BACK ? STAGE_MAX_HEAD_DIM : 1];
  __shared__ __align__(16) float gains[PAIRS == CROSSED ? STAGE_MAX_HEAD_DIM : 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int side = (int)blockIdx.x >= a.side[0].blocks ? 1 : 0;
  const RopeSide s = side ? a.side[1] : a.side[0];
  const int block = (int)blockIdx.x - (side ? a.side[0].blocks : 0);
  const int lg = a.group_log2, rows_per_pass = 32 >> lg, row = lane >> lg, unit0 = lane & ((1 << lg) - 1);
  const int half = a.rot >> 1, rest = (a.d - a.rot) >> 1;
  constexpr bool ADJ = PAIRS == ADJACENT, kCrossed = PAIRS == CROSSED;
  static_assert(!kCrossed || (NU == 1 && !FULL), "one unit per lane");
  constexpr bool kSpread = (ADJ && V > 1) || kCrossed;   // a unit's pieces lie half a row apart, so that lanes side by side take bytes side by side
  unsigned char *ring = dyn + warp * (P * kPassBytes + kTables * a.table_bytes);
  float *tables = reinterpret_cast<float *>(ring + P * kPassBytes);
  const int table_floats = a.table_bytes / 4;

  int at0[NU], at1[NU], pair[NU];   // elements of the unit's pieces, number of its first pair
  bool mine[NU], turned[NU];
  float wa[NU][V], wb[NU][V];
  pdl_enter();
#pragma unroll
  for (int n = 0; n < NU; ++n) {
    pair[n] = (unit0 + (n << lg)) * V;
    mine[n] = FULL || 2 * pair[n] < a.d;
    turned[n] = FULL || (kSpread ? half > 0 && mine[n] : pair[n] < half);   // FULL: every column turns
    if (kSpread) {
      at0[n] = pair[n];
      at1[n] = at0[n] + (a.d >> 1);
    } else if (ADJ) {
      at0[n] = 2 * pair[n];
      at1[n] = at0[n] + 1;
    } else {
      at0[n] = turned[n] ? pair[n] : a.rot + pair[n] - half;
      at1[n] = at0[n] + (turned[n] ? half : rest);
    }
    if (!kCrossed && mine[n] && s.w != nullptr) {
      Unit<T, V, ADJ> w;
      w.load(static_cast<const T *>(s.w), at0[n], at1[n]);
      w.get(wa[n], wb[n]);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) wa[n][i] = wb[n][i] = 1.f;
    }
  }
  uint32_t partner_at[V];   // where the columns' partners lie among the pieces of a pass, in bytes: 16 bits each
  auto partner = [&](int c) { return c < half ? c + half : c < a.rot ? c - half : c; };
  if (kCrossed) {
    for (int c = threadIdx.x; c < a.d; c += kThreads) gains[c] = s.w != nullptr ? to_f32<T>(static_cast<const T *>(s.w)[c]) : 1.f;
    __syncthreads();
    auto place_of = [&](int c) {
      c = mine[0] ? partner(c) : 0;
      return (row << lg) * kPieceBytes + (c < (a.d >> 1) ? c * (int)sizeof(T) : 32 * kPieceBytes + (c - (a.d >> 1)) * (int)sizeof(T));
    };
#pragma unroll
    for (int i = 0; i < V; ++i) partner_at[i] = (uint32_t)place_of(at0[0] + i) | (uint32_t)place_of(at1[0] + i) << 16;
  }
  auto partners = [&](const unsigned char *place, float (&pa)[V], float (&pb)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      pa[i] = to_f32<T>(*reinterpret_cast<const T *>(place + (partner_at[i] & 0xffff)));
      pb[i] = to_f32<T>(*reinterpret_cast<const T *>(place + (partner_at[i] >> 16)));
    }
  };
  float dwa[NU][V], dwb[NU][V];
#pragma unroll
  for (int n = 0; n < NU; ++n)
#pragma unroll
    for (int i = 0; i < V; ++i) dwa[n][i] = dwb[n][i] = 0.f;

  // this warp's part of the heads, and its tokens: t0, t0 + slots, ...
  const int wid = block * kWarps + warp, slots = s.blocks * kWarps / s.parts;
  const int part = wid % s.parts;
  const float inv_d = 1.f / (float)a.d;
  const int first = part * s.passes * rows_per_pass, heads = min(s.heads - first, s.passes * rows_per_pass);   // of this part
  const int passes = (heads + rows_per_pass - 1) / rows_per_pass;
  const int64_t t0 = wid / s.parts;
  const int64_t steps = wid < slots * s.parts && t0 < a.n ? (a.n - t0 + slots - 1) / slots * passes : 0;   // passes over all its tokens
  // a pointer goes from pass to pass, and from a token's last pass to the next token's first
  // (at the lane's first piece)
  const T *x = static_cast<const T *>(s.x) + t0 * s.x_token + (first + row) * s.x_head + at0[0];
  const T *dy = BACK ? static_cast<const T *>(s.dy) + t0 * s.dy_token + (first + row) * s.dy_head + at0[0] : nullptr;
  T *out = static_cast<T *>(s.out) + t0 * s.out_token + (first + row) * s.out_head + at0[0];
  const int64_t x_step = rows_per_pass * s.x_head, dy_step = rows_per_pass * s.dy_head, out_step = rows_per_pass * s.out_head;
  const int64_t x_jump = slots * s.x_token - passes * x_step, dy_jump = slots * s.dy_token - passes * dy_step;
  const int64_t out_jump = slots * s.out_token - passes * out_step;

  // the copies, P passes ahead of the rows in hand
  int64_t ahead_t = t0, ahead_left = steps;
  int ahead_head = 0, ahead_table = 0;   // the pass's first head
  uint32_t ahead_place = 0;
  int32_t ahead_pos = a.rot > 0 && steps > 0 ? table_row(a, t0) : 0;
  auto copy_pass = [&]() {
    if (ahead_left > 0) {
      --ahead_left;
      if (ahead_head == 0 && (FULL || a.rot > 0)) {
        float *to = tables + ahead_table * table_floats;
        const float *from = a.table + ahead_pos * a.ldt;
        if (ahead_pos < 0)
          for (int i = lane; i < a.rot; i += 32) to[i] = 0.f;
        else if (a.wide_table)
          for (int i = lane * 4; i < a.rot; i += 128) copy_piece<16>(reinterpret_cast<unsigned char *>(to + i), from + i);
        else
          for (int i = lane; i < a.rot; i += 32) copy_piece<4>(reinterpret_cast<unsigned char *>(to + i), from + i);
        if (++ahead_table == kTables) ahead_table = 0;
        ahead_t += slots;
        if (ahead_t < a.n) ahead_pos = table_row(a, ahead_t);   // known when that token begins
      }
      // a row past the last head, or a unit past D, becomes zeros: it adds nothing to a sum
      unsigned char *to = ring + ahead_place + lane * kPieceBytes;
#pragma unroll
      for (int n = 0; n < NU; ++n) {
        if (mine[n] && ahead_head + row < heads) {
          const int o0 = at0[n] - at0[0], o1 = at1[n] - at0[0];
          copy_piece<kPieceBytes>(to + n * kUnitBytes, x + o0);
          copy_piece<kPieceBytes>(to + n * kUnitBytes + 32 * kPieceBytes, x + o1);
          if (BACK) {
            copy_piece<kPieceBytes>(to + (NU + n) * kUnitBytes, dy + o0);
            copy_piece<kPieceBytes>(to + (NU + n) * kUnitBytes + 32 * kPieceBytes, dy + o1);
          }
        } else {
#pragma unroll
          for (int i = 0; i < (BACK ? 2 : 1); ++i) {
            clear_piece<kPieceBytes>(to + (i * NU + n) * kUnitBytes);
            clear_piece<kPieceBytes>(to + (i * NU + n) * kUnitBytes + 32 * kPieceBytes);
          }
        }
      }
      ahead_head += rows_per_pass;
      x += x_step;
      if (BACK) dy += dy_step;
      if (ahead_head >= heads) {
        ahead_head = 0;
        x += x_jump;
        if (BACK) dy += dy_jump;
      }
      ahead_place += kPassBytes;
      if (ahead_place == P * kPassBytes) ahead_place = 0;
    }
    asm volatile("cp.async.commit_group;\n" ::: "memory");
  };
#pragma unroll 1
  for (int i = 0; i < P; ++i) copy_pass();

  // forward: y_a = r (x_a (w_a cos) - x_b (w_b sin)), y_b = r (x_b (w_b cos) + x_a (w_a sin)); the products of the gain and the
  // angle serve all heads of the token.  backward: cosine, sine, minus sine.  CROSSED: the factors of a column and of its partner
  float ca[NU][V], cb[BACK ? 1 : NU][V], sa[NU][V], sb[NU][V];
  if (kCrossed) {   // lanes without columns
#pragma unroll
    for (int i = 0; i < V; ++i) ca[0][i] = cb[0][i] = sa[0][i] = sb[0][i] = 0.f;
  }
  int now = 0, table = 0;   // the pass's first head
  uint32_t place_at = 0;
#pragma unroll 1
  for (int64_t left = steps; left > 0; --left) {
    asm volatile("cp.async.wait_group %0;\n" ::"n"(P - 1) : "memory");
    __syncwarp();
    if (now == 0) {   // a token's first pass
      const float *cs = tables + table * table_floats;
      if (kCrossed) {
        auto factors = [&](int c, float &own, float &other) {
          const int p = c < half ? c : c - half;
          own = c < a.rot ? cs[p] : 1.f;
          other = c < a.rot ? cs[half + p] : 0.f;
          if ((c < half) != BACK) other = -other;
          if (!BACK) own *= gains[c], other *= gains[partner(c)];
        };
        if (mine[0]) {
#pragma unroll
          for (int i = 0; i < V; ++i) factors(at0[0] + i, ca[0][i], sa[0][i]), factors(at1[0] + i, cb[0][i], sb[0][i]);
        }
      }
#pragma unroll
      for (int n = 0; n < NU; ++n)
        if (!kCrossed && turned[n] && (FULL ? NU == 1 || mine[n] : mine[n])) {
          float c[V], sn[V];
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const int p = kSpread ? Unit<T, V, ADJ>::a_column(at0[n], at1[n], i) >> 1 : pair[n] + i;
            const bool turns = FULL || !kSpread || p < half;
            c[i] = turns ? cs[p] : 1.f;
            sn[i] = turns ? cs[half + p] : 0.f;
          }
          if (BACK) {
#pragma unroll
            for (int i = 0; i < V; ++i) ca[n][i] = c[i], sa[n][i] = sn[i], sb[n][i] = -sn[i];
          } else {
            v_mul(ca[n], wa[n], c);
            v_mul(cb[BACK ? 0 : n], wb[n], c);
            v_mul(sa[n], wa[n], sn);
            v_mul(sb[n], wb[n], sn);
            v_scale(sb[n], -1.f, sb[n]);
          }
        }
      if (++table == kTables) table = 0;
    }
    const bool there = now + row < heads;
    const unsigned char *place = ring + place_at + lane * kPieceBytes;
    float xa[NU][V], xb[NU][V], oa[NU][V], ob[NU][V], sq[V] = {};
#pragma unroll
    for (int n = 0; n < NU; ++n) {
      Unit<T, V, ADJ> u;
      u.take(place + n * kUnitBytes);
      u.get(xa[n], xb[n]);
      v_fma(sq, xa[n], xa[n], sq);
      v_fma(sq, xb[n], xb[n], sq);
    }
    float r = rsqrtf(fmaf(group_sum(v_total(sq), lg), inv_d, a.eps));
    if (BACK && !there) r = 0.f;   // a row that is not there: with eps = 0 its zeros would be NaN in the gains' sums
    if (!BACK) {
#pragma unroll
      for (int n = 0; n < NU; ++n) {
        v_scale(xa[n], r, xa[n]);
        v_scale(xb[n], r, xb[n]);
        if (kCrossed) {
          float pa[V], pb[V];
          partners(ring + place_at, pa, pb);
          v_scale(pa, r, pa);
          v_scale(pb, r, pb);
          v_mul(oa[n], xa[n], ca[n]);
          v_fma(oa[n], pa, sa[n], oa[n]);
          v_mul(ob[n], xb[n], cb[BACK ? 0 : n]);
          v_fma(ob[n], pb, sb[n], ob[n]);
        } else if (turned[n]) {
          v_mul(oa[n], xa[n], ca[n]);
          v_fma(oa[n], xb[n], sb[n], oa[n]);
          v_mul(ob[n], xb[n], cb[BACK ? 0 : n]);
          v_fma(ob[n], xa[n], sa[n], ob[n]);
        } else {
          v_mul(oa[n], xa[n], wa[n]);
          v_mul(ob[n], xb[n], wb[n]);
        }
      }
    } else {
      // g: the gradient turned back, times r; sums of g x w for the row and of g x for the gain
      float in[V] = {};
#pragma unroll
      for (int n = 0; n < NU; ++n) {
        Unit<T, V, ADJ> u;
        u.take(place + (NU + n) * kUnitBytes);
        float ga[V], gb[V];
        u.get(ga, gb);
        if (kCrossed) {
          float pa[V], pb[V];
          partners(ring + place_at + kUnitBytes, pa, pb);
          v_mul(ga, ga, ca[n]);
          v_fma(ga, pa, sa[n], ga);
          v_mul(gb, gb, cb[0]);
          v_fma(gb, pb, sb[n], gb);
          if (mine[n]) {
#pragma unroll
            for (int i = 0; i < V; ++i) wa[n][i] = gains[at0[n] + i], wb[n][i] = gains[at1[n] + i];
          }
        } else if (turned[n]) {
          float ta[V];
          v_mul(ta, ga, ca[n]);
          v_fma(ta, gb, sa[n], ta);
          v_mul(gb, gb, ca[n]);
          v_fma(gb, ga, sb[n], gb);
#pragma unroll
          for (int i = 0; i < V; ++i) ga[i] = ta[i];
        }
        v_scale(ga, r, ga);
        v_scale(gb, r, gb);
        v_fma(dwa[n], ga, xa[n], dwa[n]);
        v_fma(dwb[n], gb, xb[n], dwb[n]);
        v_mul(oa[n], ga, wa[n]);
        v_mul(ob[n], gb, wb[n]);
        v_fma(in, oa[n], xa[n], in);
        v_fma(in, ob[n], xb[n], in);
      }
      const float k = -(r * (r * (group_sum(v_total(in), lg) * inv_d)));   // dx = r g w - x r^2 mean(r g w x)
#pragma unroll
      for (int n = 0; n < NU; ++n) {
        v_axpy(oa[n], k, xa[n], oa[n]);
        v_axpy(ob[n], k, xb[n], ob[n]);
      }
    }
#pragma unroll
    for (int n = 0; n < NU; ++n)
      if (mine[n] && there) {
        Unit<T, V, ADJ> o;
        o.pack(oa[n], ob[n]);
        o.store(out, at0[n] - at0[0], at1[n] - at0[0]);
      }
    out += out_step;
    now += rows_per_pass;
    if (now >= heads) {
      now = 0;
      out += out_jump;
    }
    place_at += kPassBytes;
    if (place_at == P * kPassBytes) place_at = 0;
    __syncwarp();
    copy_pass();
  }

  if (BACK && s.partial != nullptr) {   // the block's share of dw: lanes of one column, then warps, always in the same order
#pragma unroll
    for (int n = 0; n < NU; ++n)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        for (int o = 16; o >= (1 << lg); o >>= 1) {
          dwa[n][i] += __shfl_xor_sync(0xffffffffu, dwa[n][i], o);
          dwb[n][i] += __shfl_xor_sync(0xffffffffu, dwb[n][i], o);
        }
        if (row == 0 && mine[n]) {
          sums[warp][Unit<T, V, ADJ>::a_column(at0[n], at1[n], i)] = dwa[n][i];
          sums[warp][Unit<T, V, ADJ>::b_column(at0[n], at1[n], i)] = dwb[n][i];
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
    if (op->ldt < op->rot_dim || op->max_pos < 1 || !aligned_to(op->table, 4)) return SSN_ERR_SHAPE;
  }
  const size_t item = op->dtype == SSN_F32 ? 4 : 2;
  if (!aligned_to(op->wq, item) || !aligned_to(op->wk, item) || !aligned_to(op->dev_status, 4)) return SSN_ERR_SHAPE;
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

// An output that starts where an input starts is that input: with other strides its rows would overwrite rows not read yet
bool other_strides(const void *out, int64_t out_token, int64_t out_head, const void *x, int64_t token, int64_t head, int64_t n, int32_t heads) {
  return heads > 0 && out == x && ((n > 1 && out_token != token) || (heads > 1 && out_head != head));
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

// The most blocks a side gets: the resident ones, dealt by a token's passes; its table row costs about one more
int side_blocks(int sms, int per_sm, int32_t heads, int32_t other, int rows_per_pass) {
  if (heads == 0) return 0;
  auto cost = [&](int32_t h) { return h == 0 ? 0 : (int64_t)(h + rows_per_pass - 1) / rows_per_pass + 1; };
  const int64_t b = (int64_t)sms * per_sm * cost(heads) / (cost(heads) + cost(other));
  return b < 1 ? 1 : (int)b;
}

template <typename T, int V, int NU, Pairs PAIRS, bool BACK, bool FULL = false>
cudaError_t launch_unit(const RopeArgs &a, cudaStream_t stream) {
  static std::atomic<uint64_t> allowed{0};
  constexpr int P = BACK ? kBackAhead : kForwardAhead;
  constexpr int kRing = kWarps * P * (BACK ? 2 : 1) * NU * 2 * 32 * V * (int)sizeof(T);
  auto kernel = qk_rope_kernel<T, V, NU, PAIRS, BACK, FULL>;
  note_kernel(STAGE_KERNEL_ROPE, V | (PAIRS == ADJACENT ? STAGE_KVAR_ADJACENT : PAIRS == CROSSED ? STAGE_KVAR_CROSSED : 0) |
                                     (FULL ? STAGE_KVAR_FULL : 0) | (BACK ? STAGE_KVAR_BACK : 0));
  const cudaError_t e = allow_dynamic_smem(kernel, kRing + kWarps * (P + 1) * STAGE_MAX_HEAD_DIM * 4, allowed);
  if (e != cudaSuccess) return e;
  return launch_dependent(kernel, (unsigned)(a.side[0].blocks + a.side[1].blocks), kThreads, kRing + kWarps * (P + 1) * a.table_bytes, stream, 1, a);
}

template <typename T, Pairs PAIRS, bool BACK>
cudaError_t launch_width(const RopeArgs &a, int v, cudaStream_t stream) {
  // whole heads that turn, with as many units as lanes, are the common case: they need no choices
  constexpr int kWide = 16 / (int)sizeof(T);
  if (v == kWide && a.rot == a.d && (a.d / (2 * kWide) & (a.d / (2 * kWide) - 1)) == 0) return launch_unit<T, kWide, 1, PAIRS, BACK, true>(a, stream);
  if constexpr (sizeof(T) == 2) {
    if (v == 8) return launch_unit<T, 8, 1, PAIRS, BACK>(a, stream);
  }
  if (v >= 4) return launch_unit<T, 4, 1, PAIRS, BACK>(a, stream);
  if (v == 2) return launch_unit<T, 2, 2, PAIRS, BACK>(a, stream);
  return launch_unit<T, 1, 4, PAIRS, BACK>(a, stream);
}

// Lanes per row and the blocks of both sides
void plan(const stage_qk_rope_t *op, RopeArgs &a, int v) {
  const int units = (op->head_dim / 2 + v - 1) / v;
  a.group_log2 = 0;
  while ((1 << a.group_log2) < units && a.group_log2 < 5) ++a.group_log2;
  const int sms = stage_sm_count(), rows = 32 >> a.group_log2;
  for (int i = 0; i < 2; ++i) plan_side(a.side[i], a.n, rows, side_blocks(sms, kPerSm, a.side[i].heads, a.side[1 - i].heads, rows));
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
  a.table_bytes = (op->rot_dim * 4 + 15) / 16 * 16;
  a.wide_table = op->rot_dim > 0 && op->rot_dim % 4 == 0 && op->ldt % 4 == 0 && aligned_to(op->table, 16);
  a.side[0].w = op->wq;
  a.side[1].w = op->wk;
}

// The width, and how pairs come together
int width_of(const stage_qk_rope_t *op, const RopeArgs &a, bool back, Pairs &pairs) {
  const size_t item = op->dtype == SSN_F32 ? 4 : 2;
  Width w(item);
  w.stride(a.d / 2);
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
  pairs = op->pairing == STAGE_PAIR_ADJACENT ? ADJACENT : HALVES;
  if (pairs == ADJACENT) return w.v;
  Width together = w;
  together.stride(a.rot / 2);
  together.stride((a.d - a.rot) / 2);
  // Units of fewer than four pairs are left to CROSSED where the rows allow wide pieces.  16384 x 40 heads of 128, bf16, 98 columns
  // turned (one pair per unit): 304 / 413 us forward and back, crossed 92 / 137; 100 columns (two) 161 / 251 and 81 / 137; 104 (four) 83 / 117
  // and 100 / 141.  The gradients take pieces of four: with eight their registers spill (183 us).
  if (together.v < 4 && w.v >= 4) {
    pairs = CROSSED;
    return back ? 4 : w.v;
  }
  return together.v;
}

template <typename T, bool BACK>
cudaError_t launch_pairs(const RopeArgs &a, Pairs pairs, int v, cudaStream_t stream) {
  if constexpr (sizeof(T) == 2 && !BACK) {
    if (pairs == CROSSED && v == 8) return launch_unit<T, 8, 1, CROSSED, BACK>(a, stream);
  }
  if (pairs == CROSSED) return launch_unit<T, 4, 1, CROSSED, BACK>(a, stream);
  return pairs == ADJACENT ? launch_width<T, ADJACENT, BACK>(a, v, stream) : launch_width<T, HALVES, BACK>(a, v, stream);
}

template <bool BACK>
ssn_status_t launch_rope(const stage_qk_rope_t *op, const RopeArgs &a, Pairs pairs, int v, cudaStream_t stream) {
  return launched(op->dtype == SSN_F32 ? launch_pairs<float, BACK>(a, pairs, v, stream) : launch_pairs<__nv_bfloat16, BACK>(a, pairs, v, stream));
}

}  // namespace
}  // namespace ssn

using namespace ssn;

extern "C" {

ssn_status_t stage_rope_table(float *table, int64_t ldt, int32_t max_pos, int32_t rot_dim, double theta, void *stream) {
  if (rot_dim < 2 || (rot_dim & 1) || max_pos < 0 || ldt < rot_dim || !(theta > 0.0) || std::isinf(theta)) return SSN_ERR_SHAPE;
  if (max_pos == 0) return SSN_OK;
  if (table == nullptr) return SSN_ERR_NULL;
  if (!aligned_to(table, 4)) return SSN_ERR_SHAPE;
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
  if (!aligned_to(pos, 4)) return SSN_ERR_SHAPE;
  if (op->rot_dim > 0 && pos == nullptr && seq_len < 1) return SSN_ERR_SHAPE;
  const int32_t d = op->head_dim;
  const size_t item = op->dtype == SSN_F32 ? 4 : 2;
  if ((st = check_heads(q, q_token, q_head, n_tokens, q_heads, d, item, false)) != SSN_OK) return st;
  if ((st = check_heads(k, k_token, k_head, n_tokens, k_heads, d, item, false)) != SSN_OK) return st;
  if ((st = check_heads(q_out, qo_token, qo_head, n_tokens, q_heads, d, item, true)) != SSN_OK) return st;
  if ((st = check_heads(k_out, ko_token, ko_head, n_tokens, k_heads, d, item, true)) != SSN_OK) return st;
  if (other_strides(q_out, qo_token, qo_head, q, q_token, q_head, n_tokens, q_heads) ||
      other_strides(k_out, ko_token, ko_head, k, k_token, k_head, n_tokens, k_heads))
    return SSN_ERR_SHAPE;
  RopeArgs a{};
  fill(op, a, pos, n_tokens, seq_len);
  const RopeSide qs{q, nullptr, q_out, op->wq, nullptr, q_token, q_head, 0, 0, qo_token, qo_head, q_heads, 0, 1, 1};
  const RopeSide ks{k, nullptr, k_out, op->wk, nullptr, k_token, k_head, 0, 0, ko_token, ko_head, k_heads, 0, 1, 1};
  a.side[0] = qs;
  a.side[1] = ks;
  Pairs pairs;
  const int v = width_of(op, a, false, pairs);
  plan(op, a, v);
  return launch_rope<false>(op, a, pairs, v, static_cast<cudaStream_t>(stream));
}

// Partial sums of at most the resident blocks, D floats each (a side never has fewer than a slot per part of its heads)
size_t stage_qk_rope_workspace_bytes(const stage_qk_rope_t *op, int64_t n_tokens, int32_t q_heads, int32_t k_heads) {
  if (check_op(op) != SSN_OK || n_tokens <= 0 || q_heads < 0 || k_heads < 0) return 0;
  const int64_t resident = (int64_t)stage_sm_count() * kPerSm + 2;
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
  if (!aligned_to(pos, 4) || !aligned_to(dwq, 4) || !aligned_to(dwk, 4)) return SSN_ERR_SHAPE;
  if (rows) {
    if (op->rot_dim > 0 && pos == nullptr && seq_len < 1) return SSN_ERR_SHAPE;
    if ((st = check_heads(dq, dq_token, dq_head, n_tokens, q_heads, d, item, false)) != SSN_OK) return st;
    if ((st = check_heads(dk, dk_token, dk_head, n_tokens, k_heads, d, item, false)) != SSN_OK) return st;
    if ((st = check_heads(q, q_token, q_head, n_tokens, q_heads, d, item, false)) != SSN_OK) return st;
    if ((st = check_heads(k, k_token, k_head, n_tokens, k_heads, d, item, false)) != SSN_OK) return st;
    if ((st = check_heads(dq_in, dqi_token, dqi_head, n_tokens, q_heads, d, item, true)) != SSN_OK) return st;
    if ((st = check_heads(dk_in, dki_token, dki_head, n_tokens, k_heads, d, item, true)) != SSN_OK) return st;
    if (other_strides(dq_in, dqi_token, dqi_head, dq, dq_token, dq_head, n_tokens, q_heads) ||
        other_strides(dk_in, dki_token, dki_head, dk, dk_token, dk_head, n_tokens, k_heads) ||
        other_strides(dq_in, dqi_token, dqi_head, q, q_token, q_head, n_tokens, q_heads) ||
        other_strides(dk_in, dki_token, dki_head, k, k_token, k_head, n_tokens, k_heads))
      return SSN_ERR_SHAPE;
    if ((dwq != nullptr || dwk != nullptr) &&
        (workspace == nullptr || !aligned_to(workspace, 16) || workspace_bytes < stage_qk_rope_workspace_bytes(op, n_tokens, q_heads, k_heads)))
      return SSN_ERR_WORKSPACE;
    fill(op, a, pos, n_tokens, seq_len);
    const RopeSide qs{q, dq, dq_in, op->wq, nullptr, q_token, q_head, dq_token, dq_head, dqi_token, dqi_head, q_heads, 0, 1, 1};
    const RopeSide ks{k, dk, dk_in, op->wk, nullptr, k_token, k_head, dk_token, dk_head, dki_token, dki_head, k_heads, 0, 1, 1};
    a.side[0] = qs;
    a.side[1] = ks;
    Pairs pairs;
    const int v = width_of(op, a, true, pairs);
    plan(op, a, v);
    float *partial = static_cast<float *>(workspace);
    if (dwq != nullptr) a.side[0].partial = partial;
    if (dwk != nullptr) a.side[1].partial = partial + (int64_t)a.side[0].blocks * d;
    if ((st = launch_rope<true>(op, a, pairs, v, s)) != SSN_OK) return st;
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
