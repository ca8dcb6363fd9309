// Distillation from a teacher's top logits: loss and gradient over rows of C logits z.
//
//   q = softmax(z / tau),  lse = log sum exp(z / tau)
//   p_j of the listed classes: softmax over the list of t / tau, or exp(t) with the rest
//   r = max(0, 1 - sum p) as one more class against the sum of q over the classes not listed
//   loss = tau^2 (sum p (log p - log q) + r (log r - log q_rest))
//   dz = dloss tau ((sum p + r) q - p)            at the listed classes (p summed over a
//   dz = dloss tau ((sum p + r) q - r q / q_rest)  class' slots), and elsewhere
//
// A list's slot whose index is no class is empty.  Where no class outside the list has a
// logit above -inf, r counts as 0.
//
// Bound by HBM: a row is read once, and once more where a gradient is written from a row that the
// registers did not hold (both in one pass over 4096 x 131072 bfloat16 488 us, 4.4 TB/s; the
// loss alone 168 us, 6.4 TB/s; the gradient alone of 999 x 50001 fp32, rows at every alignment, 89 us,
// 4.5 TB/s).  One workgroup takes a row.  A thread keeps a running maximum and the
// sum of the exponentials under it, and the workgroup joins these once.  Logits are taken from
// their maximum before anything else, so that neither a large one's digits nor a row of the
// type's lowest values are lost; a gradient by itself takes maxima and sums from the loss' pass
// (from a caller's logs of the sums alone it has what fp32 leaves of them).
//
// The listed classes are marked in a bitmap in LDS (a bit for a class, shifted like the row, so
// that a unit of 16 bytes has its own byte or half of one): a unit without one, nearly every
// unit, is summed and written whole; of the others the listed values go into a sum of their own,
// and their gradients are written by the slots' threads.  Nothing is subtracted
// from the sum of all for the rest, whose digits that would lose.
#include "internal.h"
#include "lanes.h"

#include <algorithm>
#include <cfloat>

namespace soap {
namespace {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v4u_any __attribute__((ext_vector_type(4), aligned(2)));   // 16 bytes at any element

constexpr int64_t DS_FILL = 512;          // workgroups that fill the chip
// Bytes of logits from which a call that reads them once loads past the caches (4096 x 131072 bfloat16
// loss 202 us, past them 179; gradient of 4096 x 32000 120 and 112, of 1000 x 50257 54.0 and 54.7, of
// 600 x 32000 18.7 and 22.1).  Gradients are always stored so (loss
// and gradient of 4096 x 131072 through the caches 487, past them 480, of 300 x 131072 73 and 61; gradient alone of
// 4096 x 131072 410 and 380, of 4096 x 40000 fp32 264 and 237, but of 200 MB and less, which the last cache
// may hold, 999 x 50001 fp32 70 and 86, 4096 x 32000 90 and 99; of rows read twice, 4096 x 80000 fp32, 609 and
// 623: they are not).
constexpr size_t DS_CACHED = 100 << 20;
constexpr float DS_LOG2E = 1.44269504088896340736f;

struct DsParams {
  int64_t rows, ld, ldt, ldi, ldd;
  int classes, slots, tail, t_bf16, segments;   // segments: workgroups of a row
  int wide;                               // floats of stats a row: 6, with the sums, or 2
  float tau, scale;                       // scale: log2(e) / tau
  double inv;                             // 1 / tau
  const void *z, *t;
  const int *index;
  const float *dloss;
  float *loss, *stats;
  const float *stats_in;
  void *dz;
};

enum { DS_LOSS = 1, DS_GRAD = 2 };
constexpr int DS_WIDE = 6;

// 2^x for x at or below about 0; results below 2^-126 are zeros.
__device__ __forceinline__ float ds_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

template <typename T>
constexpr int ds_vec() { return 16 / (int)sizeof(T); }
template <typename T>
__device__ __forceinline__ float ds_at(const T *p) {
  if constexpr (sizeof(T) == 4) return *p;
  else return __uint_as_float((uint32_t)*p << 16);
}
template <typename T>
__device__ __forceinline__ float ds_value(const v4u &q, int i) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(q[i]);
  else return __uint_as_float((i & 1) ? q[i / 2] & 0xffff0000u : q[i / 2] << 16);
}
template <typename T>
__device__ __forceinline__ T ds_round(float v) {
  if constexpr (sizeof(T) == 4) return v;
  else return __builtin_bit_cast(uint16_t, (__bf16)v);
}

// A row's units of 16 bytes lie where those of memory do: whole ones first .. last - 1 (the shift
// `mis` is in front of the row), and up to 2 (VEC - 1) single values in front of and behind them.
template <typename T>
struct DsRow {
  const T *z;
  int mis, first, last, front, back, edges;   // back: the column behind the whole units
  __device__ __forceinline__ DsRow(const T *row, int classes) {
    constexpr int VEC = ds_vec<T>();
    z = row;
    mis = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    first = mis ? 1 : 0;
    last = max((classes + mis) / VEC, first);
    front = min(mis ? VEC - mis : 0, classes);
    back = last * VEC - mis;
    edges = front + max(classes - max(back, front), 0);
  }
  __device__ __forceinline__ bool whole(int unit) const { return unit >= first && unit < last; }
  // Unit `at` + lane, `at` the same for all lanes: a base in scalar registers and a lane's offset.
  // FAR: past the caches.
  template <bool FAR>
  __device__ __forceinline__ v4u load(int at, uint32_t lane) const {
    const char *base = reinterpret_cast<const char *>(z) - mis * (int)sizeof(T) + (int64_t)at * 16;
    if (!whole(at + (int)lane)) return v4u(0u);
    if constexpr (FAR) return __builtin_nontemporal_load(reinterpret_cast<const v4u_any *>(base + 16 * lane));
    else return *reinterpret_cast<const v4u_any *>(base + 16 * lane);
  }
  __device__ __forceinline__ int edge(int e) const { return e < front ? e : back + e - front; }   // its column
};

// A running maximum of z and the sum of exp2((z - maximum) scale) under it; without a value
// above -inf the maximum is -inf and the sum 0 (or NaN, if there was one).
struct DsSum {
  float m, s;
};
__device__ __forceinline__ float ds_base(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ DsSum ds_join(DsSum a, DsSum b, float scale) {
  const float m = fmaxf(a.m, b.m);
  return {m, a.s * (a.m == -INFINITY ? 1.f : ds_exp2((a.m - m) * scale)) + b.s * (b.m == -INFINITY ? 1.f : ds_exp2((b.m - m) * scale))};
}
template <int NT>
__device__ __forceinline__ DsSum ds_join_all(DsSum v, float scale, DsSum *red) {
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) v = ds_join(v, {__shfl_xor(v.m, k), __shfl_xor(v.s, k)}, scale);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) v = ds_join(v, red[w], scale);
  return v;
}
// A sum from its log alone, under a logit near that log: what fp32 leaves of it.
__device__ __forceinline__ DsSum ds_from_log(float lse, float tau, double inv) {
  if (lse == -INFINITY) return {lse, 0.f};
  const float m = fminf(fmaxf((float)((double)lse * tau), -FLT_MAX), FLT_MAX);
  return {m, lse < INFINITY ? expf((float)fmin(fmax((double)lse - (double)m * inv, -60.0), 60.0)) : NAN};
}
// log s within 2^-30: s = m 2^k, log m = 2 artanh f = 2 f (1 + f^2 / 3 + f^4 / 5 ..), f = (m - 1) /
// (m + 1) of at most 0.172, of which only the first term needs more than fp32.
__device__ __forceinline__ double ds_log(float s) {
  if (!(s > 0.f && s < INFINITY)) return logf(s);
  int k = __builtin_amdgcn_frexp_expf(s);
  float m = __builtin_amdgcn_frexp_mantf(s);
  if (m < 0.70710678f) {
    m *= 2.f;
    --k;
  }
  const float r = 1.f / (m + 1.f), f = (m - 1.f) * r, z = f * f;
  const double left = ((double)m - 1.0 - f * ((double)m + 1.0)) * r;   // of f
  const float more = 2.f * f * z * (1.f / 3 + z * (0.2f + z * (1.f / 7 + z * (1.f / 9 + z * (1.f / 11)))));
  return k * 0.69314718055994530942 + 2.0 * (f + left) + more;
}
// Over a wave's lanes.
__device__ __forceinline__ double ds_total(double v) {
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) v += __shfl_xor(v, k);
  return v;
}
// What the first wave finds in the teacher's list.
struct DsList {
  float most, logs, rest, weight;         // of log p: what is taken off t, and the divisor's log; weight: of q
  int any, twice;                         // whether the list weighs anything; a class in two slots
};

// U: units of a thread that the registers hold, with workgroups that walk over rows and load the
// next one's units as they write the present one's (0: one row, read by and by, and again for the
// gradient).  The first wave sees to the list, beside the others' sums.
template <typename T, int NT, int U, int WHAT, bool FAR>
__global__ __launch_bounds__(NT) void distill_kernel(DsParams p) {
  constexpr int VEC = ds_vec<T>(), AHEAD = 4;
  constexpr bool LOSS = WHAT & DS_LOSS, GRAD = WHAT & DS_GRAD;
  extern __shared__ uint32_t map[];       // of all classes and the shift, where `marked`
  __shared__ float ps[DISTILL_MAX_SLOTS], zs[DISTILL_MAX_SLOTS];   // of the slots: log p, the student's logit,
  __shared__ int cls[DISTILL_MAX_SLOTS];                           // the class, or -1
  __shared__ DsSum red[2][NT / 64];
  __shared__ DsList list;
  const int tid = threadIdx.x;
  const bool tail = p.tail, marked = GRAD || tail, leader = __builtin_amdgcn_readfirstlane(tid >> 6) == 0;
  const float inv = (float)p.inv;
  const int words = (p.classes + VEC + 31) / 32;
  int64_t row = blockIdx.x / p.segments;
  const int segment = blockIdx.x % p.segments;
  const int64_t step = U ? gridDim.x : p.rows;
  DsRow<T> z(static_cast<const T *>(p.z) + row * p.ld, p.classes);
  // a slot of a row: class and teacher's value, and the student's logit (an empty slot: none)
  auto slot = [&](int64_t r, int j, int &c, float &t) {
    const bool in = j < p.slots;
    c = in ? p.index[r * p.ldi + j] : -1;
    t = 0.f;
    if (in) {
      if (p.t_bf16) t = ds_at(static_cast<const uint16_t *>(p.t) + r * p.ldt + j);
      else t = static_cast<const float *>(p.t)[r * p.ldt + j];
    }
  };
  auto look = [&](int &c, float &t) {
    const bool in = c >= 0 && c < p.classes;
    c = in ? c : -1;
    t = in ? t : -INFINITY;
    return in ? ds_at(z.z + c) : 0.f;
  };
  int early_c = -1;                       // the first 64, loaded ahead
  float early_t = 0.f, early_z = 0.f;
  if (leader) slot(row, tid, early_c, early_t);
  constexpr int HELD = U ? U : 1;
  v4u held[HELD];
  if constexpr (U > 0) {
#pragma unroll
    for (int u = 0; u < U; ++u) held[u] = z.template load<FAR>(u * NT, tid);
  }
  if (marked)
    for (int i = tid; i < words; i += NT) map[i] = 0u;
  __syncthreads();

#pragma unroll 1
  for (;;) {
    const int mis = z.mis;
    const int edge = z.edge(tid);         // the column of this thread's single value, where tid < z.edges
    const float single = tid < z.edges ? ds_at(z.z + edge) : 0.f;
    // ---- the teacher's list; where its classes are not needed for the sums it is looked at
    // behind these, its first 64 slots' loads before them
    if (leader) early_z = look(early_c, early_t);
    auto find = [&]() {
      DsList l = {0.f, 0.f, 0.f, 0.f, 0, 0};
      float most = -INFINITY;
      double sum = 0.0;                   // fp64: what it leaves of 1 may be little
      bool some = false, twice = false;
#pragma unroll 1
      for (int j = tid; j < p.slots; j += 64) {
        int c = early_c;
        float t = early_t, zv = early_z;
        if (j >= 64) {
          slot(row, j, c, t);
          zv = look(c, t);
        }
        most = t > most || t != t ? t : most;
        cls[j] = c;
        ps[j] = t;
        zs[j] = zv;
        if (c < 0) continue;
        some = true;
        const int b = c + mis;
        if (marked) twice |= atomicOr(&map[b >> 5], 1u << (b & 31)) >> (b & 31) & 1u;
      }
      if (!tail) l.most = ds_base(lane_reduce<64>(most, [](float a, float b) { return fmaxf(a, b); }));
#pragma unroll 1
      for (int j = tid; j < p.slots; j += 64) {
        const float t = tail ? ps[j] : (ps[j] - l.most) * inv;
        ps[j] = t;
        sum += (double)expf(t);
      }
      sum = ds_total(sum);
      l.twice = __ballot(twice) != 0;
      l.logs = tail || sum == 0.0 ? 0.f : logf((float)sum);   // p of 0 where there is nothing to divide
      // a list without a class weighs nothing, nor does one whose teacher has all of its at -inf
      l.any = tail ? __ballot(some) != 0 : sum != 0.0;
      l.rest = !tail || !l.any ? 0.f : (float)(sum == sum ? fmax(0.0, 1.0 - sum) : sum);
      l.weight = tail ? (float)sum : 1.f;
      if (tid == 0) list = l;
    };
    if (tail || !LOSS) {
      if (leader) find();
      __syncthreads();
    }

    auto bits = [&](int unit) -> uint32_t {
      return VEC == 8 ? reinterpret_cast<const uint8_t *>(map)[unit]
                      : (reinterpret_cast<const uint8_t *>(map)[unit >> 1] >> (4 * (unit & 1))) & 15u;
    };

    // ---- the student's sums: over all classes, or (tail) over those not listed and those listed
    DsSum all = {-INFINITY, 0.f}, in = {-INFINITY, 0.f};
    if constexpr (LOSS) {
      auto add = [&](DsSum &a, const float *v) {
        float m = a.m;
#pragma unroll
        for (int i = 0; i < VEC; i += 2) m = fmaxf(fmaxf(v[i], v[i + 1]), m);
        float s[2] = {0.f, 0.f};
        const float at = ds_base(m);
#pragma unroll
        for (int i = 0; i < VEC; ++i) s[i & 1] += ds_exp2((v[i] - at) * p.scale);
        if (m > a.m && a.m != -INFINITY) a.s *= ds_exp2((a.m - m) * p.scale);
        a.s += s[0] + s[1];
        a.m = m;
      };
      auto unit = [&](const v4u &q, int at) {
        float v[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = ds_value<T>(q, i);
        const uint32_t b = tail ? bits(at) : 0u;
        if (b) {
          float o[VEC];
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            o[i] = b >> i & 1u ? v[i] : -INFINITY;
            v[i] = b >> i & 1u ? -INFINITY : v[i];
          }
          add(in, o);
        }
        add(all, v);
      };
      if (tid < z.edges) {
        const int b = edge + mis;
        const DsSum one = {single, single == -INFINITY ? 0.f : single - single + 1.f};
        if (tail && map[b >> 5] >> (b & 31) & 1u) in = one;
        else all = one;
      }
      if constexpr (U > 0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (z.whole(u * NT + tid)) unit(held[u], u * NT + tid);
          __builtin_amdgcn_sched_barrier(0);   // units side by side would take the registers of others
        }
      } else {
        for (int u0 = 0; u0 < z.last; u0 += AHEAD * NT) {
          v4u q[AHEAD];
#pragma unroll
          for (int a = 0; a < AHEAD; ++a) q[a] = z.template load<FAR>(u0 + a * NT, tid);
#pragma unroll
          for (int a = 0; a < AHEAD; ++a)
            if (z.whole(u0 + a * NT + tid)) unit(q[a], u0 + a * NT + tid);
        }
      }
      if (leader && !tail) find();
      all = ds_join_all<NT>(all, p.scale, red[0]);           // its barrier is the list's too
      if (tail) in = ds_join_all<NT>(in, p.scale, red[1]);
    }
    // the sums of all classes, and with a tail those of the classes not listed
    DsSum whole = all;
    if constexpr (LOSS) {
      if (tail) whole = ds_join(all, in, p.scale);
    } else {
      const float *st = p.stats_in + p.wide * row;
      whole = p.wide == DS_WIDE ? DsSum{st[2], st[3]} : ds_from_log(st[0], p.tau, p.inv);
      all = !tail ? whole : p.wide == DS_WIDE ? DsSum{st[4], st[5]} : ds_from_log(st[1], p.tau, p.inv);
    }
    const DsList l = list;
    // no class above -inf outside the list; a sum, as logs pass fp32's range under small temperatures
    const bool alone = tail && all.s == 0.f;
    const float rest = alone ? 0.f : l.rest;

    if constexpr (LOSS) {
      if (leader) {
        double part = 0.0;                  // terms of both signs
        const float base = ds_base(whole.m);
        const double logw = ds_log(whole.s);
#pragma unroll 1
        for (int j = tid; j < p.slots; j += 64) {
          if (cls[j] < 0) continue;
          const float logp = ps[j] - l.logs, w = expf(logp);
          if (w != 0.f) part += (double)w * ((double)logp - ((double)zs[j] - base) * p.inv + logw);
        }
        part = ds_total(part);
        if (tid == 0) {
          if (rest != 0.f) {
            // log of the rest's share: both sums under their own maxima
            const double share = ((double)ds_base(all.m) - base) * p.inv + ds_log(all.s) - logw;
            part += (double)rest * (ds_log(rest) - share);
          }
          p.loss[row] = (float)(p.tau * p.tau * part);
          if (p.stats) {
            float *st = p.stats + p.wide * row;
            st[0] = fmaf(base, inv, logf(whole.s));          // log sum exp(z / tau), -inf without a value
            st[1] = tail ? fmaf(ds_base(all.m), inv, logf(all.s)) : 0.f;
            if (p.wide == DS_WIDE) {
              st[2] = whole.m;
              st[3] = whole.s;
              st[4] = tail ? all.m : 0.f;
              st[5] = tail ? all.s : 0.f;
            }
          }
        }
      }
    }
    if constexpr (!GRAD) return;

    const float g = (p.dloss ? p.dloss[row] : 1.f) * p.tau;
    const bool dead = !l.any || g == 0.f; // zeros, also where logits are no numbers
    const float weight = l.weight + rest;
    // weight q = mul_in exp2(..) with at_in; weight q - rest q / q_rest = mul exp2(..) with at, one
    // exponential under the rest's own sum
    const float at_in = ds_base(whole.m), mul_in = weight / whole.s, at = tail ? ds_base(all.m) : at_in;
    float mul = !tail ? mul_in : alone ? 0.f : (weight * ds_exp2((at - at_in) * p.scale) * (all.s / whole.s) - rest) / all.s;
    mul *= g;
    auto power = [&](float v, float under) { return ds_exp2((v - under) * p.scale); };
    T *dz = static_cast<T *>(p.dz) + row * p.ldd;
    auto put = [&](const v4u &q, int first) {    // of unit first + lane
      float v[VEC];
      if (dead) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = 0.f;
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = mul * power(ds_value<T>(q, i), at);
      }
      const uint32_t b = bits(first + tid);
      char *base = reinterpret_cast<char *>(dz) - mis * (int)sizeof(T) + (int64_t)first * 16;
      T *to = reinterpret_cast<T *>(base + 16 * (uint32_t)tid);
      v4u w;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(v[i]);
        else w[i] = (uint32_t)ds_round<T>(v[2 * i]) | (uint32_t)ds_round<T>(v[2 * i + 1]) << 16;
      }
      if (!b) {
        // past the caches, but where the row is to be read again from them
        if constexpr (U > 0 || !LOSS) __builtin_nontemporal_store(w, reinterpret_cast<v4u_any *>(to));
        else *reinterpret_cast<v4u_any *>(to) = w;
        return;
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (!(b >> i & 1u)) {
          if constexpr (sizeof(T) == 4) to[i] = v[i];
          else to[i] = (T)(w[i / 2] >> (16 * (i & 1)));
        }
    };
    if (segment == 0 && tid < z.edges) {
      const int b = edge + mis;
      if (!(map[b >> 5] >> (b & 31) & 1u)) dz[edge] = ds_round<T>(dead ? 0.f : mul * power(single, at));
    }
    const bool more = row + step < p.rows;
    // the listed classes; slots of one class write the same value
    if (leader && segment == 0) {
#pragma unroll 1
      for (int j = tid; j < p.slots; j += 64) {
        const int c = cls[j];
        if (c < 0) continue;
        float w = 0.f;
        if (l.twice) {
          for (int i = 0; i < p.slots; ++i)
            if (cls[i] == c) w += expf(ps[i] - l.logs);
        } else {
          w = expf(ps[j] - l.logs);
        }
        dz[c] = ds_round<T>(dead ? 0.f : g * (mul_in * power(zs[j], at_in) - w));
      }
    }
    const DsRow<T> zn(z.z + (more ? step * p.ld : 0), p.classes);
    if constexpr (U > 0) {
      if (more && leader) slot(row + step, tid, early_c, early_t);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (z.whole(u * NT + tid)) put(held[u], u * NT);
        if (more) held[u] = zn.template load<FAR>(u * NT, tid);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      for (int u0 = segment * AHEAD * NT; u0 < z.last; u0 += p.segments * AHEAD * NT) {
        v4u q[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) q[a] = z.template load<FAR>(u0 + a * NT, tid);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a)
          if (z.whole(u0 + a * NT + tid)) put(q[a], u0 + a * NT);
      }
    }
    if (!more) return;
    z = zn;
    row += step;
    __syncthreads();                      // the bitmap and the list are read
    for (int i = tid; i < words; i += NT) map[i] = 0u;
    __syncthreads();
  }
}

// Threads and units for a row: held in up to 128 registers of a thread by as few threads as that
// takes, with as many workgroups as the chip holds.  Loss and gradient, us (in part measured with
// stores through the caches): 4096 x 131072 bfloat16 512 threads x 32 units 503, 1024 x 16 543, read
// twice 640; 4096 x 65536 fp32 465,
// read twice 502; 8192 x 50257 bfloat16 1024 x 8 424, 512 x 16 449; 8192 x 16000 256 x 8 141, 512 x 4
// 177; 8192 x 2000 128 x 4 25, 512 x 2 34.  Longer rows are read twice, by 1024 threads (4096 x 80000
// fp32 608; 512 757, 256 826).  32 units of 512 threads are as many as fit: 233 registers in bfloat16, in fp32
// all 256 with 6 spilled (28 bytes a lane), and in both about 70 scalar ones kept in lanes of others.  Loss alone, bfloat16: workgroups side by side hide each other's
// joins, few rows need their threads (4096 x 2000: 128 threads 10.9, 256 13.0, 1024 47; 4096 x 32000:
// 256 53, 1024 75; 600 x 131072: 38 and 41; 64 x 131072: 22 and 14).  The gradient alone: 4096 x
// 2000: 128 14.2, 256 16.2; 4096 x 8000: 128 41, 256 37, 512 44, 1024 75; 600 x 32000: 20, 18.5 and 24; 2048 x 131072: 249, 228 and 220;
// 999 x 50001 fp32: 512 101, 1024 93; 200 x 50000: 17 and 20.5.
template <typename T, int WHAT>
hipError_t ds_launch(DsParams p, hipStream_t s) {
  constexpr int VEC = ds_vec<T>();
  // units wherever rows start: behind 16 bytes all at the same place, or anywhere
  const bool even = p.ld * sizeof(T) % 16 == 0 || p.rows == 1;
  const int64_t mis = even ? (int64_t)(reinterpret_cast<uintptr_t>(p.z) % 16 / sizeof(T)) : VEC - 1;
  const int64_t n = (p.classes + mis + VEC - 1) / VEC;
  const size_t lds = WHAT & DS_GRAD || p.tail ? 4 * ((p.classes + VEC + 31) / 32) : 0;
  // gradients alone need nothing of the rest of the row: few rows are cut into parts of 4096 units,
  // up to DS_FILL workgroups in all (100 x 262144 bfloat16 27 us, whole 41)
  p.segments = WHAT == DS_GRAD ? (int)std::max<int64_t>(1, std::min((n + 4095) / 4096, DS_FILL / p.rows)) : 1;
  // what no cache holds for the next pass is better kept out of them
  const bool far = (size_t)p.rows * p.classes * sizeof(T) > DS_CACHED;
#define SOAP_DS(NT, U, BLOCKS)                                                                                \
  if (U == 0 || n <= (int64_t)NT * U) {                                                                       \
    const dim3 grid((unsigned)(U ? std::min<int64_t>(p.rows, BLOCKS) : p.rows * p.segments));                 \
    constexpr bool ONCE = U == 0 && WHAT != (DS_LOSS | DS_GRAD);                                              \
    if (far && ONCE) hipLaunchKernelGGL((distill_kernel<T, NT, U, WHAT, ONCE>), grid, dim3(NT), lds, s, p);   \
    else hipLaunchKernelGGL((distill_kernel<T, NT, U, WHAT, false>), grid, dim3(NT), lds, s, p);              \
    return hipGetLastError();                                                                                 \
  }
  if constexpr (WHAT == (DS_LOSS | DS_GRAD)) {
    SOAP_DS(128, 4, 2560) SOAP_DS(256, 4, 1280) SOAP_DS(256, 8, 1024) SOAP_DS(512, 8, 512) SOAP_DS(1024, 8, 256)
    SOAP_DS(512, 32, 256)
  }
  const bool most = p.rows * 256 > UINT32_MAX;   // a launch has fewer than 2^32 threads
  if constexpr (WHAT == DS_LOSS) {
    if (n <= 1024 || most) { SOAP_DS(128, 0, 0) }
    if (n <= 4096 || p.rows >= 512) { SOAP_DS(256, 0, 0) }
  }
  if constexpr (WHAT == DS_GRAD) {
    if (n <= 256 || most) { SOAP_DS(128, 0, 0) }
    if (n <= 1024) { SOAP_DS(256, 0, 0) }
    if (n <= 8192 || p.rows < 512) { SOAP_DS(512, 0, 0) }
  }
  SOAP_DS(1024, 0, 0)
#undef SOAP_DS
}

template <int WHAT>
hipError_t ds_start(const DistillDesc &d, hipStream_t s) {
  if (d.rows <= 0) return hipSuccess;
  DsParams p{};
  p.rows = d.rows; p.ld = d.ld; p.ldt = d.ldt; p.ldi = d.ldi; p.ldd = d.ldd;
  p.classes = (int)d.classes; p.slots = (int)d.slots; p.tail = d.tail; p.t_bf16 = d.teacher_bf16;
  p.wide = d.sums ? DS_WIDE : 2;
  p.tau = d.tau; p.scale = DS_LOG2E / d.tau; p.inv = 1.0 / d.tau;
  p.z = d.logits; p.t = d.teacher; p.index = d.index; p.dloss = d.dloss;
  p.loss = d.loss; p.stats = d.stats; p.stats_in = d.stats; p.dz = d.dlogits;
  return d.bf16 ? ds_launch<uint16_t, WHAT>(p, s) : ds_launch<float, WHAT>(p, s);
}

}  // namespace

hipError_t launch_distill(const DistillDesc &d, hipStream_t s) {
  if (d.loss && d.dlogits) return ds_start<DS_LOSS | DS_GRAD>(d, s);
  return d.loss ? ds_start<DS_LOSS>(d, s) : ds_start<DS_GRAD>(d, s);
}

}  // namespace soap
