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
// lane's own values and over the lanes, then the lowest index that has it; lane j
// keeps the j-th choice.  Waves need nothing of each other on the way.
//
// The plan numbers the tokens of each expert in order.  Workgroups take chunks
// of consecutive tokens; the first launch also counts its chunk's tokens of
// each expert, the second turns the counts into each chunk's first number, the
// third gives every token its rows: of 64 tokens at a time a 64-bit mask per
// expert holds which chose it (integers: the order of the atomics does not
// matter), and a token's number is that of the bits before its own.  The sums
// of p go through per-chunk partial sums added in a fixed order.  A single
// chunk takes one launch.
//
// Bytes are few (32768 x 128 bfloat16, 8 of them: 12.6 MB, 2.4 us of HBM's time);
// the rounds of the top-k, chains of a maximum and lane exchanges, and the launches
// bound it.  Measured: a pass 22 us, in a kernel trace, which lengthens short kernels, 15 for
// the choices, 4 for the scan and 6 for the plan; 8 x 64 fp32 6.4 in the trace; the gradient of
// 32768 x 128 fp32 a pass of 16.3 us (2.2 TB/s), 17.7 in the trace.
#include "internal.h"
#include "lanes.h"

#include <algorithm>
#include <type_traits>

namespace soap {
namespace {

constexpr int RT_NT = 256;
constexpr int RT_ONE = 64;         // tokens of the single chunk of a small batch at most
constexpr int RT_CHUNK = 32;       // tokens of a chunk of a larger one at least
constexpr int RT_CHUNKS = 1024;    // chunks at most: four per thread of the second launch
constexpr int RT_MAX_E = 1024;
constexpr int RT_MAX_K = 32;

struct RtParams {
  int64_t tokens, ld, ldd, rows;
  int experts, top_k, chunk, chunks;
  int vec, vec_out;                  // logits (dlogits) can be read (written) 16 bytes at a time
  int renorm;
  float balance;
  const void *logits;
  const uint8_t *mask;
  int *index;
  float *gate;
  int *counts;
  float *loss;
  int *offsets, *position, *row_token;
  int *hist;                         // [experts + 1][RT_CHUNKS]: the last is the tokens that route
  float *psum;                       // [experts][RT_CHUNKS]
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

// The key of the value alone, of a bfloat16's key with an expert in its lower half: the
// lower bits are ones below zero, zeros above, as in the value's own key.
template <bool UNIQUE>
__device__ __forceinline__ uint32_t rt_value(uint32_t k) {
  if (!UNIQUE || k == 0u) return k;
  return (k & 0xffff0000u) | (k & 0x80000000u ? 0u : 0xffffu);
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

template <typename T, int V>
__device__ __forceinline__ void rt_store(T *row, int e0, int experts, int vec, const float *v) {
  if constexpr (sizeof(T) == 4) {
    if (vec && e0 + V <= experts) {
#pragma unroll
      for (int i = 0; i < V; i += 4)
        *reinterpret_cast<float4 *>(row + e0 + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
      return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (e0 + i < experts) row[e0 + i] = v[i];
  } else {
    uint32_t w[V / 2];
#pragma unroll
    for (int i = 0; i < V / 2; ++i)
      w[i] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * i]) |
             ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * i + 1]) << 16);
    if (vec && e0 + V <= experts) {
#pragma unroll
      for (int i = 0; i < V / 2; i += 4)
        *reinterpret_cast<uint4 *>(row + e0 + 2 * i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
      return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (e0 + i < experts) row[e0 + i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
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
  return lane_sum<LPR>(s);
}

// base[e] <- first row of expert e (each expert's rows padded to a multiple of 32),
// from the counts; offsets, if not null, gets them and the end.  Four consecutive
// experts a thread, a scan over the lanes, then over the waves.  Every thread of the
// workgroup calls it; it ends with a barrier.
__device__ void rt_offsets(const int *counts, int experts, int *base, int *offsets) {
  static_assert(RT_MAX_E == 4 * RT_NT, "four experts a thread");
  __shared__ int waves[RT_NT / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e0 = 4 * threadIdx.x;
  int n[4], sum = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    n[i] = sum;
    if (e0 + i < experts) sum += (counts[e0 + i] + 31) & ~31;
  }
  int before = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int u = __shfl_up(before, d);
    if (lane >= d) before += u;
  }
  if (lane == 63) waves[wave] = before;
  __syncthreads();
  before -= sum;
  for (int w = 0; w < wave; ++w) before += waves[w];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (e0 + i < experts) {
      base[e0 + i] = before + n[i];
      if (offsets) offsets[e0 + i] = before + n[i];
    }
  if (offsets && threadIdx.x == (experts - 1) / 4) offsets[experts] = before + sum;
  __syncthreads();
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

// balance E sum_e counts_e psum_e / (sum of counts, tokens that route): one wave.
template <typename C, typename P>
__device__ void rt_loss(const RtParams &p, C counts, P psum) {
  float f = 0.f;
  int all = 0;
  for (int e = threadIdx.x & 63; e < p.experts; e += 64) {
    f += (float)counts[e] * psum[e];
    all += counts[e];
  }
  f = lane_sum<64>(f);
  all = lane_reduce<64>(all, [](int a, int b) { return a + b; });
  if ((threadIdx.x & 63) == 0)
    p.loss[0] = all ? p.balance * (float)p.experts * f / ((float)all * (float)counts[p.experts]) : 0.f;
}

// ONE: the whole batch is one chunk and everything is done here.
template <typename T, int LPR, int V, bool ONE>
__global__ __launch_bounds__(RT_NT) void router_fwd(RtParams p) {
  constexpr bool UNIQUE = sizeof(T) == 2;            // keys with the expert's number in them
  constexpr int ROWS = RT_NT / LPR;                  // tokens of a pass
  constexpr int SLOTS = (RT_MAX_K + LPR - 1) / LPR;  // choices of a lane
  __shared__ int hist[RT_MAX_E + 1];
  __shared__ float psum[RT_NT / 64][LPR * V];
  const int tid = threadIdx.x, lane = tid % LPR, g = tid / LPR, wave = tid >> 6;
  const int e0 = lane * V, k = p.top_k;
  const int64_t t0 = (int64_t)blockIdx.x * p.chunk, t1 = min(p.tokens, t0 + p.chunk);
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
      // a bfloat16's key leaves 16 bits free: the expert, the lowest the largest
      if (UNIQUE && key[i]) key[i] = (key[i] & 0xffff0000u) | (uint32_t)(0xffff - (e0 + i));
      best = max(best, key[i]);
    }
    const uint32_t topu = lane_max<LPR>(best), top = rt_value<UNIQUE>(topu);
    const float mx = rt_unkey(top);
    const float s = rt_softmax<LPR, V>(l, e0, p.experts, top, pr);
    if (top != 0u) {
      const float inv = 1.f / s;
#pragma unroll
      for (int i = 0; i < V; ++i) acc[i] += pr[i] * inv;
      if (lane == 0) atomicAdd(&hist[p.experts], 1);
    }
    int pick[SLOTS];
    float e[SLOTS], chosen = 0.f;
    uint32_t now = topu;
#pragma unroll
    for (int slot = 0; slot < SLOTS; ++slot) {
      pick[slot] = -1;
      uint32_t mine = 0u;
      const int n = min(k - slot * LPR, LPR);
      for (int j = 0; j < n; ++j) {
        if (slot + j) {
          best = 0u;
#pragma unroll
          for (int i = 0; i < V; ++i) best = max(best, key[i]);
          now = lane_max<LPR>(best);
        }
        uint32_t at = 0x7fffffffu;               // the lowest expert that has it
        if constexpr (UNIQUE) {
          at = 0xffffu - (now & 0xffffu);
#pragma unroll
          for (int i = 0; i < V; ++i) key[i] = key[i] == now ? 0u : key[i];
        } else {
#pragma unroll
          for (int i = V - 1; i >= 0; --i) at = key[i] == now ? (uint32_t)(e0 + i) : at;
          at = lane_reduce<LPR>(at, [](uint32_t a, uint32_t b) { return min(a, b); });
#pragma unroll
          for (int i = 0; i < V; ++i) key[i] = (uint32_t)(e0 + i) == at ? 0u : key[i];
        }
        if (lane == j && now != 0u) {
          pick[slot] = (int)at;
          mine = rt_value<UNIQUE>(now);
        }
      }
      e[slot] = pick[slot] >= 0 ? expf(rt_unkey(mine) - mx) : 0.f;
      chosen += e[slot];
    }
    // a NaN of the row stays one
    const float denom = p.renorm ? (s - s) + lane_sum<LPR>(chosen) : s;
#pragma unroll
    for (int slot = 0; slot < SLOTS; ++slot) {
      const int j = slot * LPR + lane;
      if (in && j < k) {
        p.index[t * k + j] = pick[slot];
        p.gate[t * k + j] = pick[slot] >= 0 ? e[slot] / denom : 0.f;
        if (pick[slot] >= 0) atomicAdd(&hist[pick[slot]], 1);
      }
    }
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
    else p.psum[(int64_t)e * RT_CHUNKS + blockIdx.x] = v;
  }
  if constexpr (!ONE) {
    for (int e = tid; e <= p.experts; e += RT_NT) p.hist[(int64_t)e * RT_CHUNKS + blockIdx.x] = hist[e];
  } else {
    __shared__ int base[RT_MAX_E];
    __shared__ unsigned long long bits[RT_MAX_E];
    for (int e = tid; e <= p.experts; e += RT_NT) p.counts[e] = hist[e];
    __syncthreads();
    if (p.loss && wave == 0) rt_loss(p, hist, psum[0]);
    if (!p.offsets) return;                   // a plan without tokens has no other array
    rt_offsets(hist, p.experts, base, p.offsets);
    rt_assign(p, t0, t1, base, bits);
  }
}

// One expert (or, last, the tokens that route): its count, the exclusive scan of the
// chunks' counts in place, the sum of p.  Four consecutive chunks a thread.
__global__ __launch_bounds__(RT_NT) void router_scan(RtParams p) {
  static_assert(RT_CHUNKS == 4 * RT_NT, "four chunks a thread");
  __shared__ int waves[RT_NT / 64];
  __shared__ float sums[RT_NT / 64];
  const int e = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c0 = 4 * threadIdx.x;
  int *hist = p.hist + (int64_t)e * RT_CHUNKS;
  const float *psum = p.psum + (int64_t)e * RT_CHUNKS;
  const bool prob = e < p.experts;
  int n[4], sum = 0;
  float f = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    n[i] = sum;
    if (c0 + i < p.chunks) {
      sum += hist[c0 + i];
      if (prob) f += psum[c0 + i];
    }
  }
  int before = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int u = __shfl_up(before, d);
    if (lane >= d) before += u;
  }
  f = lane_sum<64>(f);
  if (lane == 63) {
    waves[wave] = before;
    sums[wave] = f;
  }
  __syncthreads();
  before -= sum;
  for (int w = 0; w < wave; ++w) before += waves[w];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (c0 + i < p.chunks) hist[c0 + i] = before + n[i];
  if (threadIdx.x == RT_NT - 1) p.counts[e] = before + sum;
  if (threadIdx.x == 0 && prob) {
    f = 0.f;
    for (int w = 0; w < RT_NT / 64; ++w) f += sums[w];
    p.ptot[e] = f;
  }
}

// Loss and offsets (workgroup 0) and the rows of every chunk's tokens.
__global__ __launch_bounds__(RT_NT) void router_plan(RtParams p) {
  __shared__ int base[RT_MAX_E];
  __shared__ unsigned long long bits[RT_MAX_E];
  if (blockIdx.x == 0 && p.loss && threadIdx.x < 64) rt_loss(p, p.counts, p.ptot);
  if (!p.offsets) return;
  rt_offsets(p.counts, p.experts, base, blockIdx.x == 0 ? p.offsets : nullptr);
  for (int e = threadIdx.x; e < p.experts; e += RT_NT) base[e] += p.hist[(int64_t)e * RT_CHUNKS + blockIdx.x];
  __syncthreads();
  const int64_t t0 = (int64_t)blockIdx.x * p.chunk, t1 = min(p.tokens, t0 + p.chunk);
  rt_assign(p, t0, t1, base, bits);
}

// A token's choices and their gradients reach the lanes that hold the experts
// through the token's own LDS, which only its lanes (of one wave) touch.
template <typename T, int LPR, int V>
__global__ __launch_bounds__(RT_NT) void router_bwd(RtParams p) {
  constexpr int ROWS = RT_NT / LPR;
  __shared__ __attribute__((aligned(16))) float dg[ROWS][LPR * V];   // dgate at the chosen experts, 0 elsewhere
  __shared__ uint32_t chosen[ROWS][LPR];     // bit i: expert lane V + i
  __shared__ int totals[RT_NT / 64];
  const int tid = threadIdx.x, lane = tid % LPR, g = tid / LPR, e0 = lane * V, k = p.top_k;
  int part = 0;
  for (int e = tid; e < p.experts; e += RT_NT) part += p.counts_in[e];
  part = lane_reduce<64>(part, [](int a, int b) { return a + b; });
  if ((tid & 63) == 0) totals[tid >> 6] = part;
#pragma unroll
  for (int i = 0; i < V; ++i) dg[g][e0 + i] = 0.f;
  chosen[g][lane] = 0u;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int w = 0; w < RT_NT / 64; ++w) total += totals[w];
  const float scale = total > 0 ? (p.dloss ? p.dloss[0] : 1.f) * p.balance * (float)p.experts /
                                      ((float)total * (float)max(1, p.counts_in[p.experts]))
                                : 0.f;
  float share[V];                            // b_e
#pragma unroll
  for (int i = 0; i < V; ++i) share[i] = e0 + i < p.experts ? scale * (float)p.counts_in[e0 + i] : 0.f;
  for (int64_t s0 = (int64_t)blockIdx.x * ROWS; s0 < p.tokens; s0 += (int64_t)gridDim.x * ROWS) {
    const int64_t t = s0 + g;
    const bool in = t < p.tokens, on = in && (!p.mask || p.mask[t]);
    float l[V], pr[V], d[V], o[V];
    rt_load<T, V>(static_cast<const T *>(p.logits) + (in ? t : s0) * p.ld, e0, p.experts, p.vec, l);
    for (int j = lane; j < k; j += LPR) {
      const int e = in ? p.index_in[t * k + j] : -1;
      if (e >= 0 && e < p.experts) {
        dg[g][e] = p.dgate ? p.dgate[t * k + j] : 0.f;
        atomicOr(&chosen[g][e / V], 1u << (e % V));
      }
    }
    __builtin_amdgcn_wave_barrier();
    const uint32_t sel = chosen[g][lane];
#pragma unroll
    for (int i = 0; i < V; ++i) d[i] = dg[g][e0 + i];
    __builtin_amdgcn_wave_barrier();
    chosen[g][lane] = 0u;
#pragma unroll
    for (int i = 0; i < V; ++i) dg[g][e0 + i] = 0.f;
    __builtin_amdgcn_wave_barrier();
    uint32_t best = 0u;
#pragma unroll
    for (int i = 0; i < V; ++i) best = max(best, on ? rt_key(l[i]) : 0u);
    const uint32_t top = lane_max<LPR>(best);
    const float inv = 1.f / rt_softmax<LPR, V>(l, e0, p.experts, top, pr);
    float s1 = 0.f;
    if (!p.renorm) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        pr[i] *= inv;
        d[i] += share[i];
        s1 = fmaf(pr[i], d[i], s1);
      }
      s1 = lane_sum<LPR>(s1);
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = pr[i] * (d[i] - s1);
    } else {
      float gs = 0.f, gd = 0.f;              // sums over the chosen of p and p dgate
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float gi = (sel >> i) & 1u ? pr[i] : 0.f;
        gs += gi;
        gd = fmaf(gi, d[i], gd);
        s1 = fmaf(pr[i], share[i], s1);
      }
      gs = lane_sum<LPR>(gs);
      gd = lane_sum<LPR>(gd);
      s1 = lane_sum<LPR>(s1) * inv;
      const float ginv = gs > 0.f ? 1.f / gs : 0.f, mean = gd * ginv;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        o[i] = pr[i] * inv * (share[i] - s1);
        if ((sel >> i) & 1u) o[i] = fmaf(pr[i] * ginv, d[i] - mean, o[i]);
      }
    }
    if (!in) continue;
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = top != 0u ? o[i] : 0.f;
    rt_store<T, V>(static_cast<T *>(p.dlogits) + t * p.ldd, e0, p.experts, p.vec_out, o);
  }
}

void rt_chunks(int64_t tokens, int *chunk, int *chunks) {
  int64_t c = RT_ONE;
  if (tokens > RT_ONE) {
    c = std::max<int64_t>(RT_CHUNK, (tokens + RT_CHUNKS - 1) / RT_CHUNKS);
    if (c > RT_CHUNK) c = (c + 63) / 64 * 64;
  }
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
  if (tokens <= RT_ONE) return 256;          // not used
  return sizeof(int) * RT_CHUNKS * (experts + 1) + sizeof(float) * (RT_CHUNKS + 1) * experts;
}

hipError_t launch_router_fwd(const RouterDesc &d, hipStream_t s) {
  RtParams p = rt_params(d);
  p.index = d.index; p.gate = d.gate; p.counts = d.counts; p.loss = d.loss;
  p.offsets = d.offsets; p.position = d.position; p.row_token = d.row_token; p.rows = d.rows;
  p.hist = static_cast<int *>(d.scratch);
  if (p.chunks > 1) {
    p.psum = reinterpret_cast<float *>(p.hist + (int64_t)RT_CHUNKS * (d.experts + 1));
    p.ptot = p.psum + (int64_t)RT_CHUNKS * d.experts;
  }
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
  hipLaunchKernelGGL(router_scan, dim3(p.experts + 1), dim3(RT_NT), 0, s, p);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(router_plan, dim3(p.offsets ? p.chunks : 1), dim3(RT_NT), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_router_bwd(const RouterDesc &d, hipStream_t s) {
  if (d.tokens <= 0) return hipSuccess;
  RtParams p = rt_params(d);
  p.index_in = d.index; p.counts_in = d.counts; p.dgate = d.dgate; p.dloss = d.dloss;
  p.dlogits = d.dlogits; p.ldd = d.ldd;
  p.vec_out = (reinterpret_cast<uintptr_t>(d.dlogits) & 15u) == 0 && d.ldd * (d.bf16 ? 2 : 4) % 16 == 0;
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
