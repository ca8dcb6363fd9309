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
// registers did not hold.  One workgroup takes a row.  A thread keeps a running maximum and the
// sum of the exponentials under it, and the workgroup joins these once.  Logits are taken from
// their maximum before anything else, so that neither a large one's digits nor a row of the
// type's lowest values are lost.
//
// The listed classes are marked in a bitmap in LDS (a bit for a class, shifted like the row, so
// that a unit of 16 bytes has its own byte or half of one): a unit without one, nearly every
// unit, is summed and written whole; of the others the listed values go into a sum of their own,
// and their gradients are written by the slots' threads.  Nothing is subtracted
// from the sum of all for the rest, whose digits that would lose.
#include "internal.h"
#include "lanes.h"

#include <algorithm>

namespace soap {
namespace {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v4u_any __attribute__((ext_vector_type(4), aligned(2)));   // 16 bytes at any element

constexpr int64_t DS_FILL = 512;          // workgroups that fill the chip
constexpr float DS_LOG2E = 1.44269504088896340736f;

struct DsParams {
  int64_t rows, ld, ldt, ldi, ldd;
  int classes, slots, tail, t_bf16, segments;   // segments: workgroups of a row
  float tau, scale;                       // scale: log2(e) / tau
  const void *z, *t;
  const int *index;
  const float *dloss;
  float *loss, *stats;
  const float *stats_in;
  void *dz;
};

enum { DS_LOSS = 1, DS_GRAD = 2 };

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

// The unit whose first value is the row's `col` (which may lie before the row or, in part,
// behind it): -inf outside.
template <typename T>
__device__ __forceinline__ v4u ds_load(const T *row, int col, int classes) {
  constexpr int VEC = ds_vec<T>();
  if (col >= 0 && col + VEC <= classes) return *reinterpret_cast<const v4u_any *>(row + col);
  v4u q;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      q[i] = col + i >= 0 && col + i < classes ? __float_as_uint(row[col + i]) : 0xff800000u;
    } else {
      const int a = col + 2 * i, b = a + 1;
      q[i] = (a >= 0 && a < classes ? (uint32_t)row[a] : 0xff80u) |
             ((b >= 0 && b < classes ? (uint32_t)row[b] : 0xff80u) << 16);
    }
  }
  return q;
}

// A running maximum of z and the sum of exp2((z - maximum) scale) under it; without a value
// above -inf the maximum is -inf and the sum 0 (or NaN, if there was one).
struct DsSum {
  float m, s;
};
__device__ __forceinline__ float ds_base(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ DsSum ds_join(DsSum a, DsSum b, float scale) {
  const float m = fmaxf(a.m, b.m);
  return {m, a.s * (a.m == -INFINITY ? 1.f : exp2f((a.m - m) * scale)) + b.s * (b.m == -INFINITY ? 1.f : exp2f((b.m - m) * scale))};
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
template <int NT, bool MAX>
__device__ __forceinline__ float ds_reduce(float v, float *red) {
  v = MAX ? lane_reduce<64>(v, [](float a, float b) { return fmaxf(a, b); }) : lane_sum<64>(v);
  __syncthreads();                        // red may still be read
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) v = MAX ? fmaxf(v, red[w]) : v + red[w];
  return v;
}

// U: units of a thread that the registers hold (0: the row is read by and by, and again for
// the gradient).
template <typename T, int NT, int U, int WHAT>
__global__ __launch_bounds__(NT) void distill_kernel(DsParams p) {
  constexpr int VEC = ds_vec<T>(), W = NT / 64, AHEAD = 4;
  constexpr bool LOSS = WHAT & DS_LOSS, GRAD = WHAT & DS_GRAD;
  extern __shared__ uint32_t map[];       // of all classes and the shift, where `marked`
  __shared__ float ps[DISTILL_MAX_SLOTS];
  __shared__ int cls[DISTILL_MAX_SLOTS];
  __shared__ float red[W];
  __shared__ DsSum red2[2][W];
  __shared__ int some, twice;
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x / p.segments;
  const int segment = blockIdx.x % p.segments;
  const T *z = static_cast<const T *>(p.z) + row * p.ld;
  const bool tail = p.tail;
  const float inv = 1.f / p.tau;
  // units lie where 16 bytes of the row do
  const int mis = (int)((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));
  const int units = (p.classes + mis + VEC - 1) / VEC;
  const bool marked = GRAD || tail;
  constexpr int HELD = U ? U : 1;
  v4u held[HELD];
  if constexpr (U > 0) {
#pragma unroll
    for (int u = 0; u < U; ++u) held[u] = ds_load<T>(z, (u * NT + tid) * VEC - mis, p.classes);
  }

  // ---- the teacher's list
  if (marked)
    for (int i = tid; i < (p.classes + mis + 31) / 32; i += NT) map[i] = 0u;
  if (tid == 0) some = twice = 0;
  float most = -INFINITY;
  for (int j = tid; j < p.slots; j += NT) {
    int c = p.index[row * p.ldi + j];
    if (c < 0 || c >= p.classes) c = -1;
    float t = -INFINITY;
    if (c >= 0) {
      t = p.t_bf16 ? ds_at(static_cast<const uint16_t *>(p.t) + row * p.ldt + j)
                   : static_cast<const float *>(p.t)[row * p.ldt + j];
    }
    cls[j] = c;
    ps[j] = t;
    most = t > most || t != t ? t : most;
  }
  __syncthreads();
  for (int j = tid; j < p.slots; j += NT) {
    if (cls[j] < 0) continue;
    some = 1;
    if (marked) {
        const int b = cls[j] + mis;
        if (atomicOr(&map[b >> 5], 1u << (b & 31)) >> (b & 31) & 1u) twice = 1;
    }
  }
  float sum = 0.f, logs = 0.f;            // of p (before it is divided), and the log of the divisor
  if (!tail) {
    most = ds_base(ds_reduce<NT, true>(most, red));
    for (int j = tid; j < p.slots; j += NT) {
      ps[j] = (ps[j] - most) * inv;
      sum += expf(ps[j]);
    }
    sum = ds_reduce<NT, false>(sum, red);
    logs = logf(sum);
  } else {
    for (int j = tid; j < p.slots; j += NT) sum += expf(ps[j]);
    sum = ds_reduce<NT, false>(sum, red);
  }
  const bool any = tail ? some : sum != 0.f;   // a list without a class weighs nothing
  float rest = !tail || !any ? 0.f : sum == sum ? fmaxf(0.f, 1.f - sum) : sum;

  auto bits = [&](int unit) -> uint32_t {
    return VEC == 8 ? reinterpret_cast<const uint8_t *>(map)[unit]
                    : (reinterpret_cast<const uint8_t *>(map)[unit >> 1] >> (4 * (unit & 1))) & 15u;
  };

  // ---- the student's sums: over all classes, or (tail) over those not listed and those listed
  DsSum all = {-INFINITY, 0.f}, in = {-INFINITY, 0.f};
  float lse = 0.f, lse_rest = 0.f;        // log sum exp(z / tau), in units of 1
  if constexpr (LOSS) {
    __syncthreads();                      // the bitmap is complete
    auto add = [&](DsSum &a, const float *v) {
      float m = v[0];
#pragma unroll
      for (int i = 1; i < VEC; ++i) m = fmaxf(m, v[i]);
      m = fmaxf(m, a.m);
      const float at = ds_base(m);
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < VEC; ++i) s += exp2f((v[i] - at) * p.scale);
      a.s = m > a.m && a.m != -INFINITY ? fmaf(a.s, exp2f((a.m - m) * p.scale), s) : a.s + s;
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
    if constexpr (U > 0) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (u * NT + tid < units) unit(held[u], u * NT + tid);
    } else {
      for (int u0 = tid; u0 < units; u0 += AHEAD * NT) {
        v4u q[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) q[a] = ds_load<T>(z, (u0 + a * NT) * VEC - mis, p.classes);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a)
          if (u0 + a * NT < units) unit(q[a], u0 + a * NT);
      }
    }
    all = ds_join_all<NT>(all, p.scale, red2[0]);
    if (tail) {
      in = ds_join_all<NT>(in, p.scale, red2[1]);
      lse_rest = fmaf(ds_base(all.m), inv, logf(all.s));      // -inf without a value
    }
  } else {
    lse = p.stats_in[2 * row];
    lse_rest = p.stats_in[2 * row + 1];
  }
  // the sums of all classes
  const DsSum whole = LOSS && tail ? ds_join(all, in, p.scale) : all;
  if constexpr (LOSS) lse = fmaf(ds_base(whole.m), inv, logf(whole.s));
  if (tail && lse_rest == -INFINITY) rest = 0.f;

  if constexpr (LOSS) {
    float part = 0.f;
    const float base = ds_base(whole.m), logw = logf(whole.s);
    for (int j = tid; j < p.slots; j += NT) {
      if (cls[j] < 0) continue;
      const float logp = tail ? ps[j] : ps[j] - logs, w = expf(logp);
      if (w != 0.f) part += w * (logp - ((ds_at(z + cls[j]) - base) * inv - logw));
    }
    part = ds_reduce<NT, false>(part, red);
    if (tid == 0) {
      if (rest != 0.f) {
        // log of the rest's share: both sums under their own maxima
        const float share = (ds_base(all.m) - base) * inv + (logf(all.s) - logw);
        part += rest * (logf(rest) - share);
      }
      p.loss[row] = p.tau * p.tau * part;
      if (p.stats) {
        p.stats[2 * row] = lse;
        p.stats[2 * row + 1] = tail ? lse_rest : 0.f;
      }
    }
  }

  if constexpr (GRAD) {
    if constexpr (!LOSS) __syncthreads(); // the bitmap is complete
    const float g = (p.dloss ? p.dloss[row] : 1.f) * p.tau;
    const bool dead = !any || g == 0.f;   // zeros, also where logits are no numbers
    const float weight = tail ? sum + rest : 1.f;
    // weight q = mul_in exp2(..) with at_in; weight q - rest q / q_rest = mul exp2(..) with at, one
    // exponential under the rest's own sum
    float at, mul, at_in, mul_in;
    if (LOSS) {
      at_in = ds_base(whole.m);
      mul_in = weight / whole.s;
      at = tail ? ds_base(all.m) : at_in;
      mul = !tail ? mul_in : lse_rest == -INFINITY ? 0.f : (weight * exp2f((at - at_in) * p.scale) * (all.s / whole.s) - rest) / all.s;
    } else {
      at_in = lse == -INFINITY ? 0.f : lse;
      mul_in = lse == -INFINITY ? NAN : weight;
      at = tail ? (lse_rest == -INFINITY ? 0.f : lse_rest) : at_in;
      mul = !tail ? mul_in : lse_rest == -INFINITY ? 0.f : weight * exp2f((lse_rest - lse) * DS_LOG2E) - rest;
    }
    mul *= g;
    // of a logit: under a maximum of logits, or under a log of sums
    auto power = [&](float v, float under) {
      return exp2f(LOSS ? (v - under) * p.scale : fmaf(v, inv, -under) * DS_LOG2E);
    };
    T *dz = static_cast<T *>(p.dz) + row * p.ldd;
    auto put = [&](const v4u &q, int at_unit) {
      const int col = at_unit * VEC - mis;
      T v[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = ds_round<T>(dead ? 0.f : mul * power(ds_value<T>(q, i), at));
      const uint32_t b = bits(at_unit);
      if (!b && col >= 0 && col + VEC <= p.classes) {
        v4u w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(v[i]);
          else w[i] = (uint32_t)v[2 * i] | (uint32_t)v[2 * i + 1] << 16;
        }
        *reinterpret_cast<v4u_any *>(dz + col) = w;
        return;
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (!(b >> i & 1u) && col + i >= 0 && col + i < p.classes) dz[col + i] = v[i];
    };
    if constexpr (U > 0) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (u * NT + tid < units) put(held[u], u * NT + tid);
    } else {
      for (int u0 = segment * AHEAD * NT + tid; u0 < units; u0 += p.segments * AHEAD * NT) {
        v4u q[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) q[a] = ds_load<T>(z, (u0 + a * NT) * VEC - mis, p.classes);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a)
          if (u0 + a * NT < units) put(q[a], u0 + a * NT);
      }
    }
    // the listed classes; slots of one class write the same value
    if (segment) return;
    for (int j = tid; j < p.slots; j += NT) {
      const int c = cls[j];
      if (c < 0) continue;
      float w = 0.f;
      if (twice) {
        for (int i = 0; i < p.slots; ++i)
          if (cls[i] == c) w += expf(tail ? ps[i] : ps[i] - logs);
      } else {
        w = expf(tail ? ps[j] : ps[j] - logs);
      }
      dz[c] = ds_round<T>(dead ? 0.f : g * (mul_in * power(ds_at(z + c), at_in) - w));
    }
  }
}

// Threads and units for a row: held in registers up to 64 of them a thread.
template <typename T, int WHAT>
hipError_t ds_launch(DsParams p, hipStream_t s) {
  const int64_t n = (p.classes + 2 * ds_vec<T>() - 2) / ds_vec<T>();   // wherever rows start
  const size_t lds = WHAT & DS_GRAD || p.tail ? 4 * ((p.classes + ds_vec<T>() + 31) / 32) : 0;
  // gradients alone need nothing of the rest of the row: few rows are cut
  p.segments = WHAT == DS_GRAD ? (int)std::max<int64_t>(1, std::min((n + 4095) / 4096, DS_FILL / p.rows)) : 1;
  const dim3 grid((unsigned)(p.rows * p.segments));
#define SOAP_DS(NT, U)                                                                     \
  if (U == 0 || n <= (int64_t)NT * U) {                                                    \
    hipLaunchKernelGGL((distill_kernel<T, NT, U, WHAT>), grid, dim3(NT), lds, s, p);         \
    return hipGetLastError();                                                              \
  }
  if constexpr (WHAT == (DS_LOSS | DS_GRAD)) { SOAP_DS(256, 4) SOAP_DS(1024, 4) SOAP_DS(1024, 8) SOAP_DS(1024, 16) }
  if (n <= 1024) { SOAP_DS(256, 0) }
  SOAP_DS(1024, 0)
#undef SOAP_DS
}

template <int WHAT>
hipError_t ds_start(const DistillDesc &d, hipStream_t s) {
  if (d.rows <= 0) return hipSuccess;
  DsParams p{};
  p.rows = d.rows; p.ld = d.ld; p.ldt = d.ldt; p.ldi = d.ldi; p.ldd = d.ldd;
  p.classes = (int)d.classes; p.slots = (int)d.slots; p.tail = d.tail; p.t_bf16 = d.teacher_bf16;
  p.tau = d.tau; p.scale = DS_LOG2E / d.tau;
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
