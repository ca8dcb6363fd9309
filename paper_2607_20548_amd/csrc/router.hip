// Router of a mixture of experts: softmax, top-k gates, per-expert counts,
// balance loss and dispatch plan of a batch of tokens, and the gradient of the
// gates and the loss.
//
//   p = softmax(l); the k largest logits of a token, ties to the lowest index
//   gate_j = p_j, or p_j over the sum of the chosen p
//   f_e = counts_e / sum of counts,  P_e = sum_t p_te / N,  loss = coef E sum_e f_e P_e
//   b_e = dloss coef E f_e / N
//   plain:         d_e = b_e + dgate_j at the chosen,  dl = p (d - sum p d)
//   renormalised:  dl = p (b - sum p b) + gate_j (dgate_j - sum gate dgate) at the chosen
//
// N is the number of tokens that route: not masked, with a logit above -inf.
// -inf and NaN logits are never chosen; a NaN makes its token's p and gates NaN.
//
// A token takes LPR lanes of a wave (8 to 64) with V = 8 or 16 consecutive
// experts each, so its logits are read once, 16 bytes per lane, and maximum and
// sum are a few lane exchanges.  A round of the top-k is a maximum over the
// lane's own values and over the lanes, and the first lane that holds it has
// the lowest index.
//
// The plan numbers the tokens of each expert in order.  Workgroups take chunks
// of consecutive tokens; the first launch also counts its chunk's tokens of
// each expert, the second turns the counts into each chunk's first number, the
// third gives every token its rows: of 64 tokens at a time a 64-bit mask per
// expert holds which chose it (integers: the order of the atomics does not
// matter), and a token's number is that of the bits before its own.  The sums
// of p go through per-chunk partial sums added in a fixed order.  A single
// chunk takes one launch.
#include "internal.h"

#include <algorithm>
#include <type_traits>

namespace soap {
namespace {

constexpr int RT_NT = 256;
constexpr int RT_CHUNK = 128;      // tokens of a chunk at least
constexpr int RT_CHUNKS = 512;     // chunks at most
constexpr int RT_MAX_E = 1024;
constexpr int RT_MAX_K = 32;
constexpr int RT_SCAN_E = 16;      // experts of a workgroup of the second launch

struct RtParams {
  int64_t tokens, ld, ldd, rows;
  int experts, top_k, chunk, chunks;
  int vec;                           // logits can be read 16 bytes at a time
  int renorm;
  float balance;
  const void *logits;
  const uint8_t *mask;
  int *index;
  float *gate;
  int *counts;
  float *loss;
  int *offsets, *position, *row_token;
  int *hist;                         // [chunks][experts + 1]: the last is the tokens that route
  float *psum;                       // [chunks][experts]
  float *ptot;                       // [experts]
  const int *index_in, *counts_in;
  const float *dgate, *dloss;
  void *dlogits;
};

// Ordered as the floats are (both zeros alike); 0 for -inf and NaN.
__device__ __forceinline__ uint32_t rt_key(float f) {
  if (!(f > -INFINITY)) return 0u;
  const uint32_t u = __float_as_uint(f + 0.f);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float rt_unkey(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}

template <int LPR>
__device__ __forceinline__ uint32_t rt_max(uint32_t v) {
#pragma unroll
  for (int m = LPR / 2; m >= 1; m >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, m));
  return v;
}
template <int LPR>
__device__ __forceinline__ float rt_sum(float v) {
#pragma unroll
  for (int m = LPR / 2; m >= 1; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

// The lane's logits e0 .. e0 + V - 1 of a row; -inf past the last expert.
template <typename T, int V>
__device__ __forceinline__ void rt_load(const T *row, int e0, int experts, int vec, float *v) {
  if (vec && e0 + V <= experts) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < V; i += 4) {
        const float4 q = *reinterpret_cast<const float4 *>(row + e0 + i);
        v[i] = q.x; v[i + 1] = q.y; v[i + 2] = q.z; v[i + 3] = q.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; i += 8) {
        const uint4 q = *reinterpret_cast<const uint4 *>(row + e0 + i);
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[i + 2 * j] = __uint_as_float(w[j] << 16);
          v[i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    v[i] = -INFINITY;
    if (e0 + i < experts) {
      if constexpr (sizeof(T) == 4) v[i] = row[e0 + i];
      else v[i] = __uint_as_float((uint32_t)row[e0 + i] << 16);
    }
  }
}

// exp(l - max) of the lane's values and their sum over the row's lanes; `top`
// is the key of the row's maximum.
template <int LPR, int V>
__device__ __forceinline__ float rt_softmax(const float *l, int e0, int experts, uint32_t top, float *p) {
  const float mx = rt_unkey(top);
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    p[i] = e0 + i < experts ? expf(l[i] - mx) : 0.f;
    s += p[i];
  }
  return rt_sum<LPR>(s);
}

// Offsets of the experts' rows (each expert's padded to a multiple of 32) from
// their counts: an inclusive scan in LDS.  Every thread of the workgroup calls it.
__device__ void rt_offsets(const int *counts, int experts, int *scan) {
  for (int e = threadIdx.x; e < experts; e += RT_NT) scan[e] = (counts[e] + 31) & ~31;
  __syncthreads();
  for (int d = 1; d < experts; d <<= 1) {
    int v[RT_MAX_E / RT_NT];
#pragma unroll
    for (int i = 0; i < RT_MAX_E / RT_NT; ++i) {
      const int e = threadIdx.x + i * RT_NT;
      v[i] = e < experts && e >= d ? scan[e - d] : 0;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < RT_MAX_E / RT_NT; ++i) {
      const int e = threadIdx.x + i * RT_NT;
      if (e < experts) scan[e] += v[i];
    }
    __syncthreads();
  }
}

// The rows of one chunk's tokens.  base[e] = first row of the chunk's tokens of
// expert e; it moves on by the tokens seen.  bits: a mask per expert.
__device__ void rt_assign(const RtParams &p, int64_t t0, int64_t t1, int *base,
                          unsigned long long *bits) {
  const int k = p.top_k;
  for (int64_t s0 = t0; s0 < t1; s0 += 64) {
    const int n = (int)min((int64_t)64, t1 - s0);
    for (int e = threadIdx.x; e < p.experts; e += RT_NT) bits[e] = 0ull;
    __syncthreads();
    for (int i = threadIdx.x; i < n * k; i += RT_NT) {
      const int e = p.index[s0 * k + i];
      if (e >= 0) atomicOr(&bits[e], 1ull << (i / k));
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n * k; i += RT_NT) {
      const int e = p.index[s0 * k + i], t = i / k;
      int row = -1;
      if (e >= 0) {
        row = base[e] + __popcll(bits[e] & ((1ull << t) - 1ull));
        p.row_token[row] = (int)(s0 + t);
      }
      p.position[s0 * k + i] = row;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.experts; e += RT_NT) base[e] += __popcll(bits[e]);
    __syncthreads();
  }
}

// ONE: the whole batch is one chunk and everything is done here.
template <typename T, int LPR, int V, bool ONE>
__global__ __launch_bounds__(RT_NT) void router_fwd(RtParams p) {
  constexpr int ROWS = RT_NT / LPR;          // tokens of a pass
  __shared__ int hist[RT_MAX_E + 1];
  __shared__ float psum[RT_NT / 64][LPR * V];
  __shared__ float denom[ROWS], rowmax[ROWS];
  __shared__ int pick[ROWS * RT_MAX_K];
  __shared__ float val[ROWS * RT_MAX_K];
  const int tid = threadIdx.x, lane = tid % LPR, g = tid / LPR, wave = tid >> 6;
  const int e0 = lane * V, k = p.top_k;
  const int64_t t0 = (int64_t)blockIdx.x * p.chunk, t1 = min(p.tokens, t0 + p.chunk);
  const uint64_t mine = (LPR == 64 ? ~0ull : ((1ull << LPR) - 1ull)) << ((tid & 63) / LPR * LPR);
  for (int e = tid; e <= p.experts; e += RT_NT) hist[e] = 0;
  if (p.row_token)                            // rows that no token takes
    for (int64_t i = (int64_t)blockIdx.x * RT_NT + tid; i < p.rows; i += (int64_t)gridDim.x * RT_NT)
      p.row_token[i] = -1;
  float acc[V];
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.f;
  __syncthreads();
  for (int64_t s0 = t0; s0 < t1; s0 += ROWS) {
    const int64_t t = s0 + g;
    const bool in = t < t1, on = in && (!p.mask || p.mask[t]);
    float l[V], pr[V];
    rt_load<T, V>(static_cast<const T *>(p.logits) + (in ? t : t0) * p.ld, e0, p.experts, p.vec, l);
    uint32_t key[V], best = 0u;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      key[i] = on ? rt_key(l[i]) : 0u;
      best = max(best, key[i]);
    }
    const uint32_t top = rt_max<LPR>(best);
    const bool routes = top != 0u;
    const float s = rt_softmax<LPR, V>(l, e0, p.experts, top, pr);
    if (routes) {
      const float inv = 1.f / s;
#pragma unroll
      for (int i = 0; i < V; ++i) acc[i] += pr[i] * inv;
      if (lane == 0) atomicAdd(&hist[p.experts], 1);
    }
    float chosen = 0.f;
    uint32_t now = top;
    for (int j = 0; j < k; ++j) {
      if (j) {
        best = 0u;
#pragma unroll
        for (int i = 0; i < V; ++i) best = max(best, key[i]);
        now = rt_max<LPR>(best);
      }
      const uint64_t who = __ballot(best == now && now != 0u) & mine;
      const bool winner = who && (int)(__ffsll((unsigned long long)who) - 1) == (tid & 63);
      if (winner) {
        int at = 0;
#pragma unroll
        for (int i = V - 1; i >= 0; --i) at = key[i] == now ? i : at;
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = i == at ? 0u : key[i];
        pick[g * RT_MAX_K + j] = e0 + at;
        val[g * RT_MAX_K + j] = rt_unkey(now);
        atomicAdd(&hist[e0 + at], 1);
      } else if (!who && lane == 0) {
        pick[g * RT_MAX_K + j] = -1;
      }
      if (now) chosen += expf(rt_unkey(now) - rt_unkey(top));
    }
    if (lane == 0) {
      rowmax[g] = rt_unkey(top);
      denom[g] = p.renorm ? (s - s) + chosen : s;      // a NaN of the row stays one
    }
    __syncthreads();
    const int n = (int)min((int64_t)ROWS, t1 - s0);
    for (int i = tid; i < n * k; i += RT_NT) {
      const int r = i / k, e = pick[r * RT_MAX_K + i - r * k];
      p.index[s0 * k + i] = e;
      p.gate[s0 * k + i] = e >= 0 ? expf(val[r * RT_MAX_K + i - r * k] - rowmax[r]) / denom[r] : 0.f;
    }
    __syncthreads();
  }
  // the chunk's sums of p: the groups of a wave, then the waves, in order
#pragma unroll
  for (int m = LPR; m < 64; m <<= 1)
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] += __shfl_xor(acc[i], m);
  if ((tid & 63) < LPR)
#pragma unroll
    for (int i = 0; i < V; ++i) psum[wave][e0 + i] = acc[i];
  __syncthreads();
  for (int e = tid; e < p.experts; e += RT_NT) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < RT_NT / 64; ++w) v += psum[w][e];
    if (ONE) psum[0][e] = v;
    else p.psum[(int64_t)blockIdx.x * p.experts + e] = v;
  }
  if constexpr (!ONE) {
    for (int e = tid; e <= p.experts; e += RT_NT)
      p.hist[(int64_t)blockIdx.x * (p.experts + 1) + e] = hist[e];
  } else {
    __shared__ int base[RT_MAX_E];
    __shared__ unsigned long long bits[RT_MAX_E];
    for (int e = tid; e <= p.experts; e += RT_NT) p.counts[e] = hist[e];
    __threadfence_block();
    __syncthreads();
    if (p.loss && wave == 0) {
      float f = 0.f;
      int all = 0;
      for (int e = tid; e < p.experts; e += 64) {
        f += (float)hist[e] * psum[0][e];
        all += hist[e];
      }
      f = rt_sum<64>(f);
#pragma unroll
      for (int m = 32; m >= 1; m >>= 1) all += __shfl_xor(all, m);
      if (tid == 0)
        p.loss[0] = all ? p.balance * (float)p.experts * f / ((float)all * (float)hist[p.experts]) : 0.f;
    }
    if (!p.row_token) return;
    rt_offsets(hist, p.experts, base);
    for (int e = tid; e <= p.experts; e += RT_NT) p.offsets[e] = e ? base[e - 1] : 0;
    __syncthreads();
    // base[e] <- first row of expert e
    for (int e = tid; e < p.experts; e += RT_NT) base[e] -= (hist[e] + 31) & ~31;
    __syncthreads();
    rt_assign(p, t0, t1, base, bits);
  }
}

// For RT_SCAN_E experts (column `experts` of hist is the tokens that route):
// counts, the exclusive scan of the chunks' counts in place, the sums of p.
// 16 slices of consecutive chunks per expert.
__global__ __launch_bounds__(RT_NT) void router_scan(RtParams p) {
  constexpr int S = RT_NT / RT_SCAN_E;
  __shared__ int tot[S][RT_SCAN_E];
  __shared__ float ps[S][RT_SCAN_E];
  const int x = threadIdx.x % RT_SCAN_E, s = threadIdx.x / RT_SCAN_E;
  const int e = blockIdx.x * RT_SCAN_E + x, E1 = p.experts + 1;
  const int per = (p.chunks + S - 1) / S;
  const int c0 = min(p.chunks, s * per), c1 = min(p.chunks, c0 + per);
  int n = 0;
  float f = 0.f;
  if (e <= p.experts) {
#pragma unroll 8
    for (int c = c0; c < c1; ++c) n += p.hist[(int64_t)c * E1 + e];
    if (e < p.experts) {
#pragma unroll 8
      for (int c = c0; c < c1; ++c) f += p.psum[(int64_t)c * p.experts + e];
    }
  }
  tot[s][x] = n;
  ps[s][x] = f;
  __syncthreads();
  if (e > p.experts) return;
  int before = 0;
  for (int i = 0; i < s; ++i) before += tot[i][x];
  if (s == S - 1) p.counts[e] = before + n;
  if (s == 0 && e < p.experts) {
    f = 0.f;
    for (int i = 0; i < S; ++i) f += ps[i][x];
    p.ptot[e] = f;
  }
  for (int c = c0; c < c1; ++c) {
    const int v = p.hist[(int64_t)c * E1 + e];
    p.hist[(int64_t)c * E1 + e] = before;
    before += v;
  }
}

// Loss and offsets (workgroup 0) and the rows of every chunk's tokens.
__global__ __launch_bounds__(RT_NT) void router_plan(RtParams p) {
  __shared__ int base[RT_MAX_E];
  __shared__ unsigned long long bits[RT_MAX_E];
  __shared__ float red[RT_NT];
  __shared__ int redn[RT_NT];
  const int tid = threadIdx.x;
  if (blockIdx.x == 0 && p.loss) {
    float f = 0.f;
    int all = 0;
    for (int e = tid; e < p.experts; e += RT_NT) {
      f += (float)p.counts[e] * p.ptot[e];
      all += p.counts[e];
    }
    red[tid] = f;
    redn[tid] = all;
    __syncthreads();
    for (int d = RT_NT / 2; d >= 1; d >>= 1) {
      if (tid < d) { red[tid] += red[tid + d]; redn[tid] += redn[tid + d]; }
      __syncthreads();
    }
    if (tid == 0)
      p.loss[0] = redn[0] ? p.balance * (float)p.experts * red[0] /
                                ((float)redn[0] * (float)p.counts[p.experts])
                          : 0.f;
  }
  if (!p.row_token) return;
  rt_offsets(p.counts, p.experts, base);
  if (blockIdx.x == 0)
    for (int e = tid; e <= p.experts; e += RT_NT) p.offsets[e] = e ? base[e - 1] : 0;
  __syncthreads();
  for (int e = tid; e < p.experts; e += RT_NT)
    base[e] += p.hist[(int64_t)blockIdx.x * (p.experts + 1) + e] - ((p.counts[e] + 31) & ~31);
  __syncthreads();
  const int64_t t0 = (int64_t)blockIdx.x * p.chunk, t1 = min(p.tokens, t0 + p.chunk);
  rt_assign(p, t0, t1, base, bits);
}

template <typename T, int LPR, int V>
__global__ __launch_bounds__(RT_NT) void router_bwd(RtParams p) {
  constexpr int ROWS = RT_NT / LPR;
  __shared__ float dg[ROWS][LPR * V];        // dgate at the chosen experts, 0 elsewhere
  __shared__ float share[LPR * V];           // b_e
  __shared__ int total;
  const int tid = threadIdx.x, lane = tid % LPR, g = tid / LPR, e0 = lane * V, k = p.top_k;
  if (tid == 0) total = 0;
  for (int i = tid; i < ROWS * LPR * V; i += RT_NT) (&dg[0][0])[i] = 0.f;
  __syncthreads();
  int part = 0;
  for (int e = tid; e < p.experts; e += RT_NT) part += p.counts_in[e];
  if (part) atomicAdd(&total, part);
  __syncthreads();
  const float scale = total > 0 ? (p.dloss ? p.dloss[0] : 1.f) * p.balance * (float)p.experts /
                                      ((float)total * (float)max(1, p.counts_in[p.experts]))
                                : 0.f;
  for (int e = tid; e < LPR * V; e += RT_NT)
    share[e] = e < p.experts ? scale * (float)p.counts_in[e] : 0.f;
  __syncthreads();
  for (int64_t s0 = (int64_t)blockIdx.x * ROWS; s0 < p.tokens; s0 += (int64_t)gridDim.x * ROWS) {
    const int64_t t = s0 + g;
    const bool in = t < p.tokens, on = in && (!p.mask || p.mask[t]);
    float l[V], pr[V];
    rt_load<T, V>(static_cast<const T *>(p.logits) + (in ? t : s0) * p.ld, e0, p.experts, p.vec, l);
    const int n = (int)min((int64_t)ROWS, p.tokens - s0) * k;
    if (p.dgate)
      for (int i = tid; i < n; i += RT_NT) {
        const int e = p.index_in[s0 * k + i];
        if (e >= 0 && e < p.experts) atomicAdd(&dg[i / k][e], p.dgate[s0 * k + i]);
      }
    __syncthreads();
    uint32_t best = 0u;
#pragma unroll
    for (int i = 0; i < V; ++i) best = max(best, on ? rt_key(l[i]) : 0u);
    const uint32_t top = rt_max<LPR>(best);
    const float inv = 1.f / rt_softmax<LPR, V>(l, e0, p.experts, top, pr);
    float o[V], s1 = 0.f;
    if (!p.renorm) {
      float d[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        pr[i] *= inv;
        d[i] = share[e0 + i] + dg[g][e0 + i];
        s1 = fmaf(pr[i], d[i], s1);
      }
      s1 = rt_sum<LPR>(s1);
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = pr[i] * (d[i] - s1);
    } else {
      // which experts were chosen: those whose index is listed
      float gs = 0.f, gd = 0.f;
      uint32_t sel = 0u;
      for (int j = 0; j < k; ++j) {
        const int e = in ? p.index_in[t * k + j] - e0 : -1;
        if (e >= 0 && e < V) sel |= 1u << e;
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float gi = (sel >> i) & 1u ? pr[i] : 0.f;
        gs += gi;
        gd = fmaf(gi, dg[g][e0 + i], gd);
        pr[i] *= inv;
        s1 = fmaf(pr[i], share[e0 + i], s1);
      }
      gs = rt_sum<LPR>(gs);
      gd = rt_sum<LPR>(gd);
      s1 = rt_sum<LPR>(s1);
      const float ginv = gs > 0.f ? 1.f / gs : 0.f, mean = gd * ginv;
      // p of the chosen back from the normalised value: gate = p / (inv gs)
      const float back = ginv / inv;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        o[i] = pr[i] * (share[e0 + i] - s1);
        if ((sel >> i) & 1u) o[i] = fmaf(pr[i] * back, dg[g][e0 + i] - mean, o[i]);
      }
    }
    if (in) {
      const bool live = top != 0u;
      T *out = static_cast<T *>(p.dlogits) + t * p.ldd;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (e0 + i < p.experts) {
          const float v = live ? o[i] : 0.f;
          if constexpr (sizeof(T) == 4) out[e0 + i] = v;
          else out[e0 + i] = __builtin_bit_cast(uint16_t, (__bf16)v);
        }
    }
    __syncthreads();
    if (p.dgate)
      for (int i = tid; i < n; i += RT_NT) {
        const int e = p.index_in[s0 * k + i];
        if (e >= 0 && e < p.experts) dg[i / k][e] = 0.f;
      }
    __syncthreads();
  }
}

void rt_chunks(int64_t tokens, int *chunk, int *chunks) {
  int64_t c = std::max<int64_t>(RT_CHUNK, (tokens + RT_CHUNKS - 1) / RT_CHUNKS);
  c = (c + 63) / 64 * 64;
  *chunk = (int)c;
  *chunks = (int)std::max<int64_t>(1, (tokens + c - 1) / c);
}

// Calls f<LPR, V>() for the experts: the fewest lanes of 8 values, 16 at most.
template <typename F>
hipError_t rt_shape(int64_t experts, F &&f) {
  if (experts <= 64) return f(std::integral_constant<int, 8>{}, std::integral_constant<int, 8>{});
  if (experts <= 128) return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 8>{});
  if (experts <= 256) return f(std::integral_constant<int, 32>{}, std::integral_constant<int, 8>{});
  if (experts <= 512) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 8>{});
  return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 16>{});
}

RtParams rt_params(const RouterDesc &d) {
  RtParams p{};
  p.tokens = d.tokens; p.experts = (int)d.experts; p.top_k = (int)d.top_k;
  p.logits = d.logits; p.ld = d.ld; p.mask = d.mask; p.renorm = d.renorm; p.balance = d.balance;
  const int elem = d.bf16 ? 2 : 4;
  p.vec = (reinterpret_cast<uintptr_t>(d.logits) & 15u) == 0 && d.ld * elem % 16 == 0;
  rt_chunks(d.tokens, &p.chunk, &p.chunks);
  return p;
}

}  // namespace

size_t router_scratch_bytes(int64_t tokens, int64_t experts) {
  int chunk, chunks;
  rt_chunks(tokens, &chunk, &chunks);
  return sizeof(int) * chunks * (experts + 1) + sizeof(float) * (chunks + 1) * experts;
}

hipError_t launch_router_fwd(const RouterDesc &d, hipStream_t s) {
  RtParams p = rt_params(d);
  p.index = d.index; p.gate = d.gate; p.counts = d.counts; p.loss = d.loss;
  p.offsets = d.offsets; p.position = d.position; p.row_token = d.row_token; p.rows = d.rows;
  p.hist = static_cast<int *>(d.scratch);
  p.psum = reinterpret_cast<float *>(p.hist + (int64_t)p.chunks * (d.experts + 1));
  p.ptot = p.psum + (int64_t)p.chunks * d.experts;
  const bool one = p.chunks == 1;
  hipError_t e = rt_shape(d.experts, [&](auto lpr, auto v) {
    constexpr int L = decltype(lpr)::value, V = decltype(v)::value;
    const dim3 grid((unsigned)p.chunks);
    if (d.bf16) {
      if (one) hipLaunchKernelGGL((router_fwd<uint16_t, L, V, true>), grid, dim3(RT_NT), 0, s, p);
      else hipLaunchKernelGGL((router_fwd<uint16_t, L, V, false>), grid, dim3(RT_NT), 0, s, p);
    } else {
      if (one) hipLaunchKernelGGL((router_fwd<float, L, V, true>), grid, dim3(RT_NT), 0, s, p);
      else hipLaunchKernelGGL((router_fwd<float, L, V, false>), grid, dim3(RT_NT), 0, s, p);
    }
    return hipGetLastError();
  });
  if (e != hipSuccess || one) return e;
  hipLaunchKernelGGL(router_scan, dim3((p.experts + RT_SCAN_E) / RT_SCAN_E), dim3(RT_NT), 0, s, p);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(router_plan, dim3(p.row_token ? p.chunks : 1), dim3(RT_NT), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_router_bwd(const RouterDesc &d, hipStream_t s) {
  if (d.tokens <= 0) return hipSuccess;
  RtParams p = rt_params(d);
  p.index_in = d.index; p.counts_in = d.counts; p.dgate = d.dgate; p.dloss = d.dloss;
  p.dlogits = d.dlogits; p.ldd = d.ldd;
  return rt_shape(d.experts, [&](auto lpr, auto v) {
    constexpr int L = decltype(lpr)::value, V = decltype(v)::value;
    const int64_t rows = RT_NT / L;
    const dim3 grid((unsigned)std::min<int64_t>((d.tokens + rows - 1) / rows, 2048));
    if (d.bf16) hipLaunchKernelGGL((router_bwd<uint16_t, L, V>), grid, dim3(RT_NT), 0, s, p);
    else hipLaunchKernelGGL((router_bwd<float, L, V>), grid, dim3(RT_NT), 0, s, p);
    return hipGetLastError();
  });
}

}  // namespace soap
