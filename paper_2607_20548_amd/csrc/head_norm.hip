// RMS norm of every head of queries and keys and the rotation by its token's position,
// forward and backward.
//
//   r = 1 / sqrt(sum x^2 / D + eps),  h = x r,  y = R (w h)
//   g = R^T dy,  dx = r (w g - h sum(w g h) / D),  dw = sum over tokens and heads of g h
//
// R turns the pairs (a, b) of a head's first `rot` values by the token's angles
// position * frequency: (a cos - b sin, b cos + a sin).  Pairs are values of the same index
// in both halves of the turned part, or neighbours; the values past it are paired alike and
// turned by 0.  Sums and statistics are fp32, outputs are rounded once.
//
// An angle reaches 2^31 radians and more, where fp32 (and fp64 of a product rounded to
// radians) has no digits left of the turn: it is formed in fp64 in half turns, brought to
// [-1, 1] there, and only then rounded for fp32 sine and cosine.
//
// Bound by HBM (2 and 3 values moved per element): LANES lanes of a wave hold a head, each
// UNITS x VEC pairs (16 bytes of either half, or 32 bytes of neighbours), so that the
// rotation stays within a lane, and the 64 / LANES groups of a wave take different heads of
// one token, whose angles are formed once for all of them, or where a token has few heads a
// token each.  16384 tokens of 16 + 16 heads of 128 bfloat16: 50 us forward (5.4 TB/s), 89 backward
// (4.5 TB/s, with 5 for the second kernel).  Away from such heads lanes idle (halves of 72 take 16
// lanes of 9: 81 and 154, floor 58 and 87) or units are partial and go value by value (rotary 36 of 128: 150
// and 321).  Backward, sums for both sides, a head and its gradient take 209 to 241 registers in bfloat16 (two
// waves a SIMD; fp32 132 to 197, three or two), and 14 to 54 scalar ones are kept in lanes of others.
//
// dw: every workgroup walks over tokens and writes the sums over its own, a second kernel adds
// these in a fixed order.
#include "internal.h"
#include "lanes.h"

#include <algorithm>

namespace soap {
namespace {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v4u_any __attribute__((ext_vector_type(4), aligned(2)));   // 16 bytes at any element

constexpr int HN_THREADS = 256, HN_WAVES = HN_THREADS / 64;
// Workgroups backward, and rows of partial sums: two for every compute unit (the size above: 256
// 119 us, 512 95, 1024 100, before the angles were shared).
constexpr int64_t HN_BLOCKS_BWD = 512;
// Waves that fill the chip: fewer tokens share their heads out over several (300 tokens of 64 + 64
// heads of 256 fp32: 1 wave a token 45.6 us forward and 75 backward, up to 1024 waves 21 and 38, 4096
// 15.3 and 31, 16384 16.9 and 34).
constexpr int64_t HN_FEW = 4096;
// Bytes of heads from which their loads go past the caches, where a half is whole lines (16384 tokens of
// 16 + 16 heads of 128 bfloat16: 56 and 51 us forward, 95 and 93 backward; 8192 of fp32 56 and 47, 83 and
// 79; 3000 of bfloat16 13.5 and 14.5; halves of 64 bytes, 16384 of 64: 31.4 and 34.7).
constexpr int64_t HN_CACHED = 60 << 20;
constexpr int HN_FIN = 1024, HN_FIN_COLS = 32;

struct HnSide {                          // queries or keys
  const void *x, *dy;
  void *out;
  const float *w;
  int heads, chunks;                     // chunks of heads that a wave takes at once
  int64_t xt, xh, dt, dh, ot, oh;        // strides of tokens and heads
};
struct HnParams {
  int64_t tokens, tasks;
  int dim, rot, split;
  HnSide side[2];
  float eps;
  const int *pos;
  const double *freq;
  float *part;                           // [workgroup][2][dim]
};

template <typename T>
constexpr int hn_vec() { return 16 / (int)sizeof(T); }

// n of VEC values from p on, zeros after them.  FAR: past the caches.
template <typename T, bool FAR>
__device__ __forceinline__ v4u hn_load(const T *p, int n) {
  if (n == hn_vec<T>()) {
    if constexpr (FAR) return __builtin_nontemporal_load(reinterpret_cast<const v4u_any *>(p));
    else return *reinterpret_cast<const v4u_any *>(p);
  }
  v4u q = v4u(0u);
#pragma unroll
  for (int i = 0; i < hn_vec<T>(); ++i)
    if (i < n) {
      if constexpr (sizeof(T) == 4) q[i] = __float_as_uint(p[i]);
      else q[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
    }
  return q;
}
template <typename T>
__device__ __forceinline__ float hn_value(const v4u &q, int i) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(q[i]);
  else return __uint_as_float((i & 1) ? q[i / 2] & 0xffff0000u : q[i / 2] << 16);
}
template <typename T>
__device__ __forceinline__ void hn_store(T *p, int n, const float *v) {
  v4u q;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) q[i] = __float_as_uint(v[i]);
    else
      q[i] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * i]) |
             ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * i + 1]) << 16);
  }
  if (n == hn_vec<T>()) {
    *reinterpret_cast<v4u_any *>(p) = q;
    return;
  }
#pragma unroll
  for (int i = 0; i < hn_vec<T>(); ++i)
    if (i < n) {
      if constexpr (sizeof(T) == 4) p[i] = v[i];
      else p[i] = (uint16_t)(q[i / 2] >> (16 * (i & 1)));
    }
}

// The VEC pairs of a lane's unit: columns of its two 16 bytes, how many values of each are
// the head's, and where its frequencies are.
struct HnUnit {
  int c0, c1, n0, n1, turn, turned;      // turned: pairs with a frequency
};
template <int VEC, bool NEAR>
__device__ __forceinline__ HnUnit hn_unit(const HnParams &p, int u) {
  const int half = p.rot / 2, rest = (p.dim - p.rot) / 2, first = (half + VEC - 1) / VEC;
  const bool in = u < first;             // the pairs that are turned, then the others
  const int at = (in ? u : u - first) * VEC, n = min(max((in ? half : rest) - at, 0), VEC);
  HnUnit r;
  if (NEAR) {
    r.c0 = (in ? 0 : p.rot) + 2 * at;
    r.c1 = r.c0 + VEC;
    r.n0 = min(2 * n, VEC);
    r.n1 = 2 * n - r.n0;
  } else {
    r.c0 = (in ? 0 : p.rot) + at;
    r.c1 = r.c0 + (in ? half : rest);
    r.n0 = r.n1 = n;
  }
  r.turn = at;
  r.turned = in ? n : 0;
  return r;
}

// a[i], b[i]: the pairs in two loads.
template <typename T, bool NEAR>
__device__ __forceinline__ void hn_pairs(const v4u &q0, const v4u &q1, float *a, float *b) {
  constexpr int VEC = hn_vec<T>();
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    if constexpr (NEAR) {
      a[i] = 2 * i < VEC ? hn_value<T>(q0, (2 * i) % VEC) : hn_value<T>(q1, (2 * i) % VEC);
      b[i] = 2 * i < VEC ? hn_value<T>(q0, (2 * i) % VEC + 1) : hn_value<T>(q1, (2 * i) % VEC + 1);
    } else {
      a[i] = hn_value<T>(q0, i);
      b[i] = hn_value<T>(q1, i);
    }
  }
}
template <typename T, bool NEAR>
__device__ __forceinline__ void hn_put(T *row, const HnUnit &u, const float *a, const float *b) {
  constexpr int VEC = hn_vec<T>();
  if constexpr (NEAR) {
    float v[2 * VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      v[2 * i] = a[i];
      v[2 * i + 1] = b[i];
    }
    hn_store<T>(row + u.c0, u.n0, v);
    hn_store<T>(row + u.c1, u.n1, v + VEC);
  } else {
    hn_store<T>(row + u.c0, u.n0, a);
    hn_store<T>(row + u.c1, u.n1, b);
  }
}
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));
template <int VEC>
__device__ __forceinline__ void hn_floats(const float *w, int n, float *v) {   // ones past n
#pragma unroll
  for (int i = 0; i < VEC; ++i) v[i] = 1.f;
  if (n == VEC) {
#pragma unroll
    for (int i = 0; i < VEC; i += 4) {
      const v4f_any q = *reinterpret_cast<const v4f_any *>(w + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i + j] = q[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (i < n) v[i] = w[i];
  }
}
template <int VEC, bool NEAR>
__device__ __forceinline__ void hn_weights(const float *w, const HnUnit &u, float *a, float *b) {
  float lo[VEC], hi[VEC];
  hn_floats<VEC>(w + u.c0, w ? u.n0 : 0, lo);
  hn_floats<VEC>(w + u.c1, w ? u.n1 : 0, hi);
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    a[i] = !NEAR ? lo[i] : 2 * i < VEC ? lo[(2 * i) % VEC] : hi[(2 * i) % VEC];
    b[i] = !NEAR ? hi[i] : 2 * i < VEC ? lo[(2 * i) % VEC + 1] : hi[(2 * i) % VEC + 1];
  }
}

__device__ __forceinline__ float2 hn_turn(double position, double frequency) {
  double t = position * frequency * 0.31830988618379067154;      // 1 / pi: half turns
  t -= 2.0 * rint(0.5 * t);
  float2 r;
  sincospif((float)t, &r.y, &r.x);
  return r;
}
// Cosine and sine of the token's pairs.  Where the wave has one token they are formed once, one a
// lane, and handed to the lanes through LDS (`own`: the wave's); a lane's own token's by itself.
template <int VEC, int UNITS, bool EACH>
__device__ __forceinline__ void hn_angles(const HnParams &p, const HnUnit *un, int64_t token, float2 *own,
                                          float (*c)[VEC], float (*s)[VEC]) {
  const double pos = p.pos ? (double)p.pos[token] : (double)token;
  if constexpr (EACH) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float2 v = i < un[u].turned ? hn_turn(pos, p.freq[un[u].turn + i]) : make_float2(1.f, 0.f);
        c[u][i] = v.x;
        s[u][i] = v.y;
      }
    return;
  }
  const int half = p.rot / 2;
  __builtin_amdgcn_wave_barrier();               // what was there is read
  for (int i = threadIdx.x & 63; i < half; i += 64) own[i] = hn_turn(pos, p.freq[i]);
  __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int u = 0; u < UNITS; ++u)
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const bool in = i < un[u].turned;
      const float2 v = own[in ? un[u].turn + i : 0];
      c[u][i] = in ? v.x : 1.f;
      s[u][i] = in ? v.y : 0.f;
    }
}

// Chunks of heads in turn: those of the queries, then those of the keys.  A wave's slots take
// heads of one token, or (EACH) the same heads of a token each.
template <typename T, int LANES, int UNITS, bool NEAR, bool EACH, bool FAR>
struct HnHeads {
  static constexpr int SLOTS = 64 / LANES, IT = UNITS == 1 ? 2 : 1, STEP = EACH ? 1 : SLOTS, MANY = IT * STEP;
  v4u q[IT][UNITS][2];
  __device__ __forceinline__ void load(const T *x, int64_t stride, int heads, int part, int slot, const HnUnit *un) {
#pragma unroll
    for (int j = 0; j < IT; ++j) {
      const T *row = x + (int64_t)min(part * MANY + (EACH ? 0 : slot) + j * STEP, heads - 1) * stride;
#pragma unroll
      for (int u = 0; u < UNITS; ++u) {
        q[j][u][0] = hn_load<T, FAR>(row + un[u].c0, un[u].n0);
        q[j][u][1] = hn_load<T, FAR>(row + un[u].c1, un[u].n1);
      }
    }
  }
};

template <typename T, int LANES, int UNITS, bool NEAR, bool EACH, bool FAR>
__global__ __launch_bounds__(HN_THREADS) void head_norm_fwd(HnParams p) {
  using Heads = HnHeads<T, LANES, UNITS, NEAR, EACH, FAR>;
  constexpr int VEC = hn_vec<T>(), IT = Heads::IT, STEP = Heads::STEP, MANY = Heads::MANY;
  constexpr int TOKENS = EACH ? Heads::SLOTS : 1;            // of a wave
  __shared__ float2 angle[HN_WAVES][LANES * UNITS * VEC];
  const int lane = threadIdx.x % LANES, slot = threadIdx.x % 64 / LANES;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t task = (int64_t)blockIdx.x * HN_WAVES + wave;
  if (task >= p.tasks) return;
  const int64_t group = task / p.split, mine = group * TOKENS + (EACH ? slot : 0), token = min(mine, p.tokens - 1);
  const HnSide d0 = p.side[0], d1 = p.side[1];
  const int all = d0.chunks + d1.chunks;
  HnUnit un[UNITS];
#pragma unroll
  for (int u = 0; u < UNITS; ++u) un[u] = hn_unit<VEC, NEAR>(p, u * LANES + lane);
  auto fetch = [&](Heads &to, int at) {
    const bool k = at >= d0.chunks;
    to.load(static_cast<const T *>(k ? d1.x : d0.x) + token * (k ? d1.xt : d0.xt), k ? d1.xh : d0.xh,
            k ? d1.heads : d0.heads, at - (k ? d0.chunks : 0), slot, un);
  };
  int at = (int)(task - group * p.split);
  Heads now, next;
  fetch(now, at);
  float co[UNITS][VEC], si[UNITS][VEC];
  hn_angles<VEC, UNITS, EACH>(p, un, token, angle[wave], co, si);
  const float inv = 1.f / (float)p.dim;
#pragma unroll 1
  for (; at < all; at += p.split) {
    if (at + p.split < all) fetch(next, at + p.split);
    const bool k = at >= d0.chunks;
    const int heads = k ? d1.heads : d0.heads, h0 = (at - (k ? d0.chunks : 0)) * MANY + (EACH ? 0 : slot);
    T *y = static_cast<T *>(k ? d1.out : d0.out) + token * (k ? d1.ot : d0.ot);
    const int64_t oh = k ? d1.oh : d0.oh;
    float wa[UNITS][VEC], wb[UNITS][VEC];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) hn_weights<VEC, NEAR>(k ? d1.w : d0.w, un[u], wa[u], wb[u]);
#pragma unroll
    for (int j = 0; j < IT; ++j) {
      float a[UNITS][VEC], b[UNITS][VEC], sum = 0.f;
#pragma unroll
      for (int u = 0; u < UNITS; ++u) {
        hn_pairs<T, NEAR>(now.q[j][u][0], now.q[j][u][1], a[u], b[u]);
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum = fmaf(a[u][i], a[u][i], fmaf(b[u][i], b[u][i], sum));
      }
      const float r = 1.f / sqrtf(lane_sum<LANES>(sum) * inv + p.eps);
      const int h = h0 + j * STEP;
      if (h >= heads || mine >= p.tokens) continue;
#pragma unroll
      for (int u = 0; u < UNITS; ++u) {
        float ya[VEC], yb[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float ha = a[u][i] * r * wa[u][i], hb = b[u][i] * r * wb[u][i];
          ya[i] = ha * co[u][i] - hb * si[u][i];
          yb[i] = hb * co[u][i] + ha * si[u][i];
        }
        hn_put<T, NEAR>(y + (int64_t)h * oh, un[u], ya, yb);
      }
    }
    now = next;
  }
}

// out: dx (none if null); part: the sums of g h over the workgroup's tokens (none if null).
template <typename T, int LANES, int UNITS, bool NEAR, bool EACH, bool FAR>
__global__ __launch_bounds__(HN_THREADS) void head_norm_bwd(HnParams p) {
  using Heads = HnHeads<T, LANES, UNITS, NEAR, EACH, FAR>;
  constexpr int VEC = hn_vec<T>(), IT = Heads::IT, STEP = Heads::STEP, MANY = Heads::MANY;
  constexpr int TOKENS = EACH ? Heads::SLOTS : 1;            // of a wave
  __shared__ float red[HN_WAVES][LANES * UNITS * VEC * 4];
  float2 *angle = reinterpret_cast<float2 *>(red[threadIdx.x >> 6]);   // twice as many places as pairs
  const int lane = threadIdx.x % LANES, slot = threadIdx.x % 64 / LANES;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const HnSide d0 = p.side[0], d1 = p.side[1];
  const int all = d0.chunks + d1.chunks;
  HnUnit un[UNITS];
  float dw[2][UNITS][2][VEC];
#pragma unroll
  for (int u = 0; u < UNITS; ++u) {
    un[u] = hn_unit<VEC, NEAR>(p, u * LANES + lane);
#pragma unroll
    for (int i = 0; i < VEC; ++i) dw[0][u][0][i] = dw[0][u][1][i] = dw[1][u][0][i] = dw[1][u][1][i] = 0.f;
  }
  const float inv = 1.f / (float)p.dim;
  const int64_t stride = (int64_t)gridDim.x * HN_WAVES;
  int64_t task = (int64_t)blockIdx.x * HN_WAVES + wave, group = task / p.split;
  int at = (int)(task - group * p.split);
  Heads x, dy;
  auto fetch = [&](Heads &tx, Heads &td, int64_t tok, int c) {
    const bool k = c >= d0.chunks;
    const int part = c - (k ? d0.chunks : 0), heads = k ? d1.heads : d0.heads;
    tx.load(static_cast<const T *>(k ? d1.x : d0.x) + tok * (k ? d1.xt : d0.xt), k ? d1.xh : d0.xh, heads, part, slot, un);
    td.load(static_cast<const T *>(k ? d1.dy : d0.dy) + tok * (k ? d1.dt : d0.dt), k ? d1.dh : d0.dh, heads, part, slot, un);
  };
  float co[UNITS][VEC], si[UNITS][VEC];
  bool fresh = true;                             // the angles are another token's
#pragma unroll 1
  while (task < p.tasks) {
    const int64_t mine = group * TOKENS + (EACH ? slot : 0), now = min(mine, p.tokens - 1);
    fetch(x, dy, now, at);
    if (fresh) hn_angles<VEC, UNITS, EACH>(p, un, now, angle, co, si);
    const int c = at;
    at += p.split;
    fresh = at >= all;
    if (fresh) {
      task += stride;
      group = task / p.split;
      at = (int)(task - group * p.split);
    }
    const bool k = c >= d0.chunks;
    const int heads = k ? d1.heads : d0.heads, h0 = (c - (k ? d0.chunks : 0)) * MANY + (EACH ? 0 : slot);
    T *dx = static_cast<T *>(k ? d1.out : d0.out);
    const bool wanted = dx != nullptr;
    dx += now * (k ? d1.ot : d0.ot);
    const int64_t oh = k ? d1.oh : d0.oh;
    float wa[UNITS][VEC], wb[UNITS][VEC];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) hn_weights<VEC, NEAR>(k ? d1.w : d0.w, un[u], wa[u], wb[u]);
    auto process = [&](float (&sums)[UNITS][2][VEC]) {
#pragma unroll
      for (int j = 0; j < IT; ++j) {
        const int h = h0 + j * STEP;
        float a[UNITS][VEC], b[UNITS][VEC], ga[UNITS][VEC], gb[UNITS][VEC], sum = 0.f, dot = 0.f;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
          hn_pairs<T, NEAR>(x.q[j][u][0], x.q[j][u][1], a[u], b[u]);
#pragma unroll
          for (int i = 0; i < VEC; ++i) sum = fmaf(a[u][i], a[u][i], fmaf(b[u][i], b[u][i], sum));
        }
        const float r = 1.f / sqrtf(lane_sum<LANES>(sum) * inv + p.eps);
        const bool live = h < heads && mine < p.tokens;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
          float ea[VEC], eb[VEC];
          hn_pairs<T, NEAR>(dy.q[j][u][0], dy.q[j][u][1], ea, eb);
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            a[u][i] *= r;
            b[u][i] *= r;
            const float ta = ea[i] * co[u][i] + eb[i] * si[u][i], tb = eb[i] * co[u][i] - ea[i] * si[u][i];
            if (live) {
              sums[u][0][i] = fmaf(ta, a[u][i], sums[u][0][i]);
              sums[u][1][i] = fmaf(tb, b[u][i], sums[u][1][i]);
            }
            ga[u][i] = ta * wa[u][i];
            gb[u][i] = tb * wb[u][i];
            dot = fmaf(ga[u][i], a[u][i], fmaf(gb[u][i], b[u][i], dot));
          }
        }
        dot = lane_sum<LANES>(dot) * inv;
        if (!live || !wanted) continue;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            ga[u][i] = r * (ga[u][i] - a[u][i] * dot);
            gb[u][i] = r * (gb[u][i] - b[u][i] * dot);
          }
          hn_put<T, NEAR>(dx + (int64_t)h * oh, un[u], ga[u], gb[u]);
        }
      }
    };
    if (k) process(dw[1]);
    else process(dw[0]);
  }
  if (!p.part) return;
  __syncthreads();                               // the angles' place is free
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
#pragma unroll
      for (int ab = 0; ab < 2; ++ab)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          float v = dw[k][u][ab][i];
#pragma unroll
          for (int m = LANES; m < 64; m <<= 1) v += __shfl_xor(v, m);
          if (slot == 0) red[wave][((k * UNITS + u) * 2 + ab) * VEC * LANES + i * LANES + lane] = v;
        }
  __syncthreads();
  if (wave != 0 || slot != 0) return;
  float *part = p.part + (int64_t)blockIdx.x * 2 * p.dim;
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
#pragma unroll
      for (int ab = 0; ab < 2; ++ab)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const int at = NEAR ? 2 * i + ab : i, n = NEAR ? un[u].n0 + un[u].n1 : un[u].n0;
          if (at >= n) continue;
          float v = 0.f;
#pragma unroll
          for (int w = 0; w < HN_WAVES; ++w) v += red[w][((k * UNITS + u) * 2 + ab) * VEC * LANES + i * LANES + lane];
          part[k * p.dim + (!NEAR && ab ? un[u].c1 : un[u].c0) + at] = v;
        }
}

// The sums of the workgroups' rows, 32 columns of the queries' and keys' weights at a time.
__global__ __launch_bounds__(HN_FIN) void head_norm_finish(const float *part, int blocks, int dim, float *dq, float *dk) {
  constexpr int C = HN_FIN_COLS, S = HN_FIN / C;
  __shared__ float red[HN_FIN];
  const int at = blockIdx.x * C + threadIdx.x % C, s = threadIdx.x / C;
  float v = 0.f;
  if (at < 2 * dim)
#pragma unroll 16
    for (int b = s; b < blocks; b += S) v += part[(int64_t)b * 2 * dim + at];
  red[threadIdx.x] = v;
  __syncthreads();
  if (s != 0 || at >= 2 * dim) return;
#pragma unroll
  for (int k = 1; k < S; ++k) v += red[k * C + threadIdx.x];
  if (at < dim && dq) dq[at] = v;
  if (at >= dim && dk) dk[at - dim] = v;
}

struct HnShape {
  int lanes, units;
  bool each, far;
};
// Lanes of a head, and whether a wave's slots take a token each: where its steps are fewer by
// a quarter, the heads of one token leaving slots idle (60000 tokens of 1 + 1 heads of 128 bfloat16:
// 20 us, slots for heads 73).
HnShape hn_shape(const HeadNormDesc &d) {
  const int64_t vec = d.bf16 ? 8 : 4, half = d.rotary / 2, rest = (d.dim - d.rotary) / 2;
  const int64_t n = (half + vec - 1) / vec + (rest + vec - 1) / vec;
  HnShape r{n <= 4 ? 4 : n <= 8 ? 8 : n <= 16 ? 16 : n <= 32 ? 32 : 64, n <= 64 ? 1 : 2, false, false};
  const int64_t slots = 64 / r.lanes, it = r.units == 1 ? 2 : 1, q = d.side[0].heads, k = d.side[1].heads;
  auto steps = [&](int64_t each) { return (q + each - 1) / each + (k + each - 1) / each; };
  const int64_t e = d.bf16 ? 2 : 4;
  r.far = d.rotary == d.dim && d.dim / 2 * e % 128 == 0 && d.tokens * (q + k) * d.dim * e > HN_CACHED;
  r.each = slots > 1 && 5 * steps(it) * ((d.tokens + slots - 1) / slots) < 4 * steps(it * slots) * d.tokens;
  return r;
}
int64_t hn_blocks_bwd(int64_t tasks) { return std::min((tasks + HN_WAVES - 1) / HN_WAVES, HN_BLOCKS_BWD); }

HnParams hn_params(const HeadNormDesc &d, const HnShape &sh) {
  HnParams p{};
  p.tokens = d.tokens; p.dim = (int)d.dim; p.rot = (int)d.rotary; p.eps = d.eps;
  p.pos = d.positions; p.freq = d.frequencies;
  const int slots = 64 / sh.lanes, each = (sh.each ? 1 : slots) * (sh.units == 1 ? 2 : 1);
  const int64_t groups = sh.each ? (d.tokens + slots - 1) / slots : d.tokens;
  for (int k = 0; k < 2; ++k) {
    const HeadNormSide &a = d.side[k];
    HnSide &b = p.side[k];
    b.x = a.x; b.dy = a.dy; b.out = a.out; b.w = a.weight;
    b.heads = (int)a.heads; b.chunks = (int)((a.heads + each - 1) / each);
    b.xt = a.x_token; b.xh = a.x_head; b.dt = a.dy_token; b.dh = a.dy_head; b.ot = a.out_token; b.oh = a.out_head;
  }
  const int64_t chunks = p.side[0].chunks + p.side[1].chunks;
  p.split = (int)std::max<int64_t>(1, std::min(chunks, HN_FEW / std::max<int64_t>(groups, 1)));
  p.tasks = chunks ? groups * p.split : 0;
  return p;
}

template <bool BWD, typename T, bool NEAR>
hipError_t hn_launch(const HnParams &p, const HnShape &sh, hipStream_t s) {
  const int64_t blocks = BWD ? hn_blocks_bwd(p.tasks) : (p.tasks + HN_WAVES - 1) / HN_WAVES;
#define SOAP_HN_FAR(L, U, E, F)                                                                                  \
  if (sh.lanes == L && sh.units == U && sh.each == E) {                                                          \
    if constexpr (BWD) hipLaunchKernelGGL((head_norm_bwd<T, L, U, NEAR, E, F>), dim3((unsigned)blocks), dim3(HN_THREADS), 0, s, p); \
    else hipLaunchKernelGGL((head_norm_fwd<T, L, U, NEAR, E, F>), dim3((unsigned)blocks), dim3(HN_THREADS), 0, s, p); \
    return hipGetLastError();                                                                                    \
  }
#define SOAP_HN(L, U, E) SOAP_HN_FAR(L, U, E, false)
  if constexpr (!NEAR) {
    if (sh.far) {
      SOAP_HN_FAR(8, 1, false, true) SOAP_HN_FAR(16, 1, false, true) SOAP_HN_FAR(32, 1, false, true)
      if constexpr (sizeof(T) == 4) { SOAP_HN_FAR(64, 1, false, true) }
    }
  }
  SOAP_HN(4, 1, false) SOAP_HN(8, 1, false) SOAP_HN(16, 1, false) SOAP_HN(32, 1, false) SOAP_HN(64, 1, false)
  SOAP_HN(4, 1, true) SOAP_HN(8, 1, true) SOAP_HN(16, 1, true) SOAP_HN(32, 1, true)
  if constexpr (sizeof(T) == 4) { SOAP_HN(64, 2, false) }
#undef SOAP_HN
#undef SOAP_HN_FAR
  return hipErrorInvalidValue;
}

template <bool BWD>
hipError_t hn_start(const HeadNormDesc &d, const HnParams &p, const HnShape &sh, hipStream_t s) {
  if (!p.tasks) return hipSuccess;
  if (d.bf16) return d.near ? hn_launch<BWD, uint16_t, true>(p, sh, s) : hn_launch<BWD, uint16_t, false>(p, sh, s);
  return d.near ? hn_launch<BWD, float, true>(p, sh, s) : hn_launch<BWD, float, false>(p, sh, s);
}

}  // namespace

// Rows of partial sums as many as a backward pass has workgroups at most.
size_t head_norm_part_bytes(int64_t tokens, int64_t dim) {
  return tokens ? sizeof(float) * 2 * dim * HN_BLOCKS_BWD : 0;
}

hipError_t launch_head_norm_fwd(const HeadNormDesc &d, hipStream_t s) {
  const HnShape sh = hn_shape(d);
  return hn_start<false>(d, hn_params(d, sh), sh, s);
}

hipError_t launch_head_norm_bwd(const HeadNormDesc &d, hipStream_t s) {
  const HnShape sh = hn_shape(d);
  HnParams p = hn_params(d, sh);
  const bool sums = d.side[0].dweight || d.side[1].dweight;
  p.part = sums ? d.part : nullptr;
  const hipError_t e = hn_start<true>(d, p, sh, s);
  if (e != hipSuccess || !sums) return e;
  hipLaunchKernelGGL(head_norm_finish, dim3((unsigned)((2 * d.dim + HN_FIN_COLS - 1) / HN_FIN_COLS)), dim3(HN_FIN), 0, s,
                     p.part, p.tasks ? (int)hn_blocks_bwd(p.tasks) : 0, p.dim, d.side[0].dweight, d.side[1].dweight);
  return hipGetLastError();
}

}  // namespace soap
