// Layer norm of the rows of a matrix, forward and backward.
//
//   mu = sum x / C,  var = sum (x - mu)^2 / C,  r = 1 / sqrt(var + eps)
//   h = (x - mu) r,  y = w h + b
//   g = w dy,  dx = r (g - mean(g) - h mean(g h)),  dw = sum_rows dy h,  db = sum_rows dy
//
// All statistics and sums are fp32; a bfloat16 output is rounded once.
//
// Both are bound by HBM (2 and 3 values moved per element), so a row is read
// once: a group of GROUP threads (8 lanes to a workgroup) holds it in
// registers, V values per thread, and takes the mean, the centred sum of
// squares and, backward, the two dot products from there.  Unit u of a thread
// covers the VEC consecutive columns from (u GROUP + thread) VEC on, VEC values
// being 16 bytes where the operands allow it and one otherwise.  Workgroups
// walk over the rows and keep the weight (and the sums of dw, db over their
// rows) in registers.
//
// dw and db: every workgroup writes the sums over its rows, a second kernel
// adds these partial sums in a fixed order, so results do not vary between
// runs.
#include "internal.h"

#include <algorithm>

namespace soap {
namespace {

constexpr int64_t LN_BLOCKS_FWD = 2048;  // workgroups of a forward launch at most
constexpr int64_t LN_BLOCKS_BWD = 512;   // of a backward launch: rows of partial sums
constexpr int LN_FIN = 1024;             // threads of the second kernel: 64 columns x 16 slices

struct LnParams {
  int64_t rows;
  int cols;
  const void *x, *dy;
  int64_t ldx, lddy, ldo;
  const float *w, *b;
  const float *mean_in, *rstd_in;
  float eps;
  void *out;
  float *mean, *rstd;
  float *part;   // [workgroup][2][cols]: dw, db
};

__device__ __forceinline__ float ln_bf16(uint32_t h) { return __uint_as_float(h << 16); }

template <typename T, int VEC>
__device__ __forceinline__ void ln_load(const T *p, float *v) {
  if constexpr (sizeof(T) == 4 && VEC == 4) {
    const float4 q = *reinterpret_cast<const float4 *>(p);
    v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
  } else if constexpr (sizeof(T) == 2 && VEC == 8) {
    const uint4 q = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = ln_bf16(w[i] & 0xffffu);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else if constexpr (sizeof(T) == 2) {
    v[0] = ln_bf16(*reinterpret_cast<const uint16_t *>(p));
  } else {
    v[0] = *reinterpret_cast<const float *>(p);
  }
}

template <typename T, int VEC>
__device__ __forceinline__ void ln_store(T *p, const float *v) {
  if constexpr (sizeof(T) == 4 && VEC == 4) {
    *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
  } else if constexpr (sizeof(T) == 2 && VEC == 8) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * i]) |
             ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * i + 1]) << 16);
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint16_t *>(p) = __builtin_bit_cast(uint16_t, (__bf16)v[0]);
  } else {
    *reinterpret_cast<float *>(p) = v[0];
  }
}

template <int VEC>
__device__ __forceinline__ void ln_param(const float *p, int col, int cols, float dflt, float *v) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) v[i] = p && col + i < cols ? p[col + i] : dflt;
}

// Sum over the GROUP threads of a row, in a fixed tree; every one of them gets
// it.  `red` has a slot for each wave and is used by one call between barriers.
template <int GROUP>
__device__ __forceinline__ float ln_sum(float v, float *red) {
  constexpr int W = GROUP < 64 ? GROUP : 64;
#pragma unroll
  for (int m = W / 2; m >= 1; m >>= 1) v += __shfl_xor(v, m);
  if constexpr (GROUP > 64) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[wave] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < GROUP / 64; ++i) v += red[i];
  }
  return v;
}

template <int GROUP>
constexpr int ln_threads() { return GROUP < 256 ? 256 : GROUP; }

template <typename T, int VEC, int GROUP, int V>
__global__ __launch_bounds__(ln_threads<GROUP>()) void layer_norm_fwd(LnParams p) {
  constexpr int NT = ln_threads<GROUP>(), ROWS = NT / GROUP, U = V / VEC;
  __shared__ float red[NT / 64];
  const int lane = threadIdx.x % GROUP, g = threadIdx.x / GROUP;
  const float inv = 1.f / (float)p.cols;
  float w[U][VEC], b[U][VEC];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int col = (u * GROUP + lane) * VEC;
    ln_param<VEC>(p.w, col, p.cols, 1.f, w[u]);
    ln_param<VEC>(p.b, col, p.cols, 0.f, b[u]);
  }
  const int64_t step = (int64_t)gridDim.x * ROWS;
  for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < p.rows; r0 += step) {
    const int64_t row = r0 + g;
    const bool live = row < p.rows;
    const T *x = static_cast<const T *>(p.x) + (live ? row : p.rows - 1) * p.ldx;
    float v[U][VEC];
    float s = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int col = (u * GROUP + lane) * VEC;
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[u][i] = 0.f;
      if (col < p.cols) ln_load<T, VEC>(x + col, v[u]);
#pragma unroll
      for (int i = 0; i < VEC; ++i) s += v[u][i];
    }
    const float mu = ln_sum<GROUP>(s, red) * inv;
    s = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if ((u * GROUP + lane) * VEC < p.cols) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          v[u][i] -= mu;
          s = fmaf(v[u][i], v[u][i], s);
        }
      }
    }
    const float r = 1.f / sqrtf(ln_sum<GROUP>(s, red) * inv + p.eps);
    if (!live) continue;
    T *y = static_cast<T *>(p.out) + row * p.ldo;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int col = (u * GROUP + lane) * VEC;
      if (col >= p.cols) continue;
      float o[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) o[i] = fmaf(v[u][i] * r, w[u][i], b[u][i]);
      ln_store<T, VEC>(y + col, o);
    }
    if (lane == 0) {
      if (p.mean) p.mean[row] = mu;
      if (p.rstd) p.rstd[row] = r;
    }
  }
}

// out = dx (none if null); part = the sums of dy h and dy over the workgroup's
// rows (none if null).
template <typename T, int VEC, int GROUP, int V>
__global__ __launch_bounds__(ln_threads<GROUP>()) void layer_norm_bwd(LnParams p) {
  constexpr int NT = ln_threads<GROUP>(), ROWS = NT / GROUP, U = V / VEC;
  __shared__ float red[NT / 64];
  const int lane = threadIdx.x % GROUP, g = threadIdx.x / GROUP;
  const float inv = 1.f / (float)p.cols;
  float w[U][VEC], dw[U][VEC], db[U][VEC];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    ln_param<VEC>(p.w, (u * GROUP + lane) * VEC, p.cols, 1.f, w[u]);
#pragma unroll
    for (int i = 0; i < VEC; ++i) dw[u][i] = db[u][i] = 0.f;
  }
  const int64_t step = (int64_t)gridDim.x * ROWS;
  for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < p.rows; r0 += step) {
    const int64_t row = r0 + g;
    const bool live = row < p.rows;
    const int64_t at = live ? row : p.rows - 1;
    const T *x = static_cast<const T *>(p.x) + at * p.ldx;
    const T *dy = static_cast<const T *>(p.dy) + at * p.lddy;
    const float mu = p.mean_in[at], r = p.rstd_in[at];
    float h[U][VEC], d[U][VEC];
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int col = (u * GROUP + lane) * VEC;
#pragma unroll
      for (int i = 0; i < VEC; ++i) h[u][i] = d[u][i] = 0.f;
      if (col < p.cols && live) {
        ln_load<T, VEC>(x + col, h[u]);
        ln_load<T, VEC>(dy + col, d[u]);
#pragma unroll
        for (int i = 0; i < VEC; ++i) h[u][i] = (h[u][i] - mu) * r;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        db[u][i] += d[u][i];
        dw[u][i] = fmaf(d[u][i], h[u][i], dw[u][i]);
        d[u][i] *= w[u][i];
        s1 += d[u][i];
        s2 = fmaf(d[u][i], h[u][i], s2);
      }
    if (!p.out) continue;
    s1 = ln_sum<GROUP>(s1, red) * inv;
    s2 = ln_sum<GROUP>(s2, red) * inv;
    if (!live) continue;
    T *dx = static_cast<T *>(p.out) + row * p.ldo;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int col = (u * GROUP + lane) * VEC;
      if (col >= p.cols) continue;
      float o[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) o[i] = r * (d[u][i] - s1 - h[u][i] * s2);
      ln_store<T, VEC>(dx + col, o);
    }
  }
  if (!p.part) return;
  float *part = p.part + (int64_t)blockIdx.x * 2 * p.cols;
  if constexpr (GROUP < 64) {      // the groups of a wave
#pragma unroll
    for (int m = GROUP; m < 64; m <<= 1)
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          dw[u][i] += __shfl_xor(dw[u][i], m);
          db[u][i] += __shfl_xor(db[u][i], m);
        }
  }
  if constexpr (GROUP <= 64) {     // the waves, in order
    __shared__ float sum[2][GROUP * V];
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int k = 0; k < NT / 64; ++k) {
      if (wave == k && (threadIdx.x & 63) < GROUP) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            const int c = (u * GROUP + lane) * VEC + i;
            sum[0][c] = k == 0 ? dw[u][i] : sum[0][c] + dw[u][i];
            sum[1][c] = k == 0 ? db[u][i] : sum[1][c] + db[u][i];
          }
      }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < p.cols; c += NT) {
      part[c] = sum[0][c];
      part[p.cols + c] = sum[1][c];
    }
  } else {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const int c = (u * GROUP + lane) * VEC + i;
        if (c >= p.cols) continue;
        part[c] = dw[u][i];
        part[p.cols + c] = db[u][i];
      }
  }
}

// dw[c] or db[c] (by blockIdx.y) = sum over the workgroups' partial sums:
// slice s of 16 adds workgroups s, s + 16, ... in order, then the slices in
// order.
__global__ __launch_bounds__(LN_FIN) void layer_norm_bwd_finish(const float *__restrict__ part,
                                                               int nb, int cols,
                                                               float *__restrict__ dw,
                                                               float *__restrict__ db) {
  __shared__ float red[LN_FIN];
  float *out = blockIdx.y == 0 ? dw : db;
  if (!out) return;
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), s = threadIdx.x >> 6;
  float v = 0.f;
  if (c < cols) {
    const float *src = part + (int64_t)blockIdx.y * cols + c;
#pragma unroll 8
    for (int k = s; k < nb; k += LN_FIN / 64) v += src[(int64_t)k * 2 * cols];
  }
  red[threadIdx.x] = v;
  __syncthreads();
  if (s != 0 || c >= cols) return;
  for (int k = 1; k < LN_FIN / 64; ++k) v += red[k * 64 + threadIdx.x];
  out[c] = v;
}

bool ln_aligned(const void *p, int64_t ld, int elem) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * elem % 16 == 0;
}

// Threads per row and values per thread: the fewest threads of a wave that
// hold the row in at most 32 values each, whole workgroups past 2048 columns.
struct LnShape {
  int group, v;
};
LnShape ln_shape(int64_t cols) {
  if (cols <= 256) return {8, cols <= 64 ? 8 : cols <= 128 ? 16 : 32};
  if (cols <= 2048) return {64, cols <= 512 ? 8 : cols <= 1024 ? 16 : 32};
  if (cols <= 8192) return {256, cols <= 4096 ? 16 : 32};
  return {512, 32};
}

int64_t ln_blocks(int64_t rows, int64_t cols, int64_t most) {
  const int group = ln_shape(cols).group;
  const int64_t per = group < 256 ? 256 / group : 1;
  return std::min((rows + per - 1) / per, most);
}

template <bool BWD, typename T, int VEC>
hipError_t ln_launch(const LnParams &p, hipStream_t s) {
  const LnShape sh = ln_shape(p.cols);
  const dim3 grid((unsigned)ln_blocks(p.rows, p.cols, BWD ? LN_BLOCKS_BWD : LN_BLOCKS_FWD));
#define SOAP_LN(G, N)                                                                             \
  if (sh.group == G && sh.v == N) {                                                               \
    if constexpr (BWD)                                                                            \
      hipLaunchKernelGGL((layer_norm_bwd<T, VEC, G, N>), grid, dim3(ln_threads<G>()), 0, s, p);   \
    else                                                                                          \
      hipLaunchKernelGGL((layer_norm_fwd<T, VEC, G, N>), grid, dim3(ln_threads<G>()), 0, s, p);   \
    return hipGetLastError();                                                                     \
  }
  SOAP_LN(8, 8) SOAP_LN(8, 16) SOAP_LN(8, 32)
  SOAP_LN(64, 8) SOAP_LN(64, 16) SOAP_LN(64, 32)
  SOAP_LN(256, 16) SOAP_LN(256, 32) SOAP_LN(512, 32)
#undef SOAP_LN
  return hipErrorInvalidValue;
}

template <bool BWD>
hipError_t ln_dispatch(const LnParams &p, bool bf16, bool wide, hipStream_t s) {
  if (bf16) return wide ? ln_launch<BWD, uint16_t, 8>(p, s) : ln_launch<BWD, uint16_t, 1>(p, s);
  return wide ? ln_launch<BWD, float, 4>(p, s) : ln_launch<BWD, float, 1>(p, s);
}

}  // namespace

size_t layer_norm_part_bytes(int64_t rows, int64_t cols) {
  return sizeof(float) * 2 * cols * ln_blocks(rows, cols, LN_BLOCKS_BWD);
}

hipError_t launch_layer_norm_fwd(const LayerNormDesc &d, hipStream_t s) {
  if (d.rows <= 0) return hipSuccess;
  LnParams p{};
  p.rows = d.rows; p.cols = (int)d.cols;
  p.x = d.x; p.ldx = d.ldx; p.w = d.weight; p.b = d.bias; p.eps = d.eps;
  p.out = d.out; p.ldo = d.ldo; p.mean = d.mean; p.rstd = d.rstd;
  const int elem = d.bf16 ? 2 : 4;
  const bool wide = d.cols * elem % 16 == 0 && ln_aligned(d.x, d.ldx, elem) &&
                    ln_aligned(d.out, d.ldo, elem);
  return ln_dispatch<false>(p, d.bf16, wide, s);
}

hipError_t launch_layer_norm_bwd(const LayerNormDesc &d, hipStream_t s) {
  LnParams p{};
  p.rows = d.rows; p.cols = (int)d.cols;
  p.x = d.x; p.ldx = d.ldx; p.dy = d.dy; p.lddy = d.lddy; p.w = d.weight;
  p.mean_in = d.mean; p.rstd_in = d.rstd; p.out = d.out; p.ldo = d.ldo;
  p.part = d.dweight || d.dbias ? d.part : nullptr;
  const int elem = d.bf16 ? 2 : 4;
  const bool wide = d.cols * elem % 16 == 0 && ln_aligned(d.x, d.ldx, elem) &&
                    ln_aligned(d.dy, d.lddy, elem) && (!d.out || ln_aligned(d.out, d.ldo, elem));
  hipError_t e = hipSuccess;
  if (d.rows > 0 && (e = ln_dispatch<true>(p, d.bf16, wide, s)) != hipSuccess) return e;
  if (!p.part) return hipSuccess;
  hipLaunchKernelGGL(layer_norm_bwd_finish, dim3((unsigned)((d.cols + 63) / 64), 2), dim3(LN_FIN),
                     0, s, p.part, (int)ln_blocks(d.rows, d.cols, LN_BLOCKS_BWD), p.cols, d.dweight,
                     d.dbias);
  return hipGetLastError();
}

}  // namespace soap
