// Layer norm of the rows of a matrix, forward and backward.
//
//   mu = sum x / C,  var = sum (x - mu)^2 / C,  r = 1 / sqrt(var + eps)
//   h = (x - mu) r,  y = w h + b
//   g = w dy,  dx = r (g - mean(g) - h mean(g h)),  dw = sum_rows dy h,  db = sum_rows dy
//
// All statistics and sums are fp32; a bfloat16 output is rounded once.
//
// Both are bound by HBM (2 and 3 values moved per element), so a row is read
// once: a group of GROUP threads (8 lanes to a workgroup) holds it in registers, V
// values per thread, and takes the mean, the centred sum of squares and,
// backward, the two dot products from there.  Unit u of a thread covers the VEC
// consecutive columns from (u GROUP + thread) VEC on, 16 bytes, read and written at
// once wherever the whole unit is inside the row (rows need no alignment past that
// of an element) and value by value in the unit that crosses its end.  Workgroups
// walk over the rows, keep the weight (and the sums of dw, db over their rows) in
// registers and load their next row before they reduce the present one.
//
// Groups of a whole workgroup meet once per row: the variance is put together from
// the waves' own means and squares about them.  Measured: 16384 x 4096 bfloat16 53 us a
// pass forward (5.1 TB/s; a copy of 1 GiB reaches 5.2) and 81 backward (in a kernel trace
// 78, 5.2 TB/s, and 5 for the second kernel), without the row ahead and with two meetings
// 76 and 103.  Rows that start between two 16 bytes are slower: 16384 x 2048 bfloat16 27 us
// forward and 45 backward, x 2047 44 and 70.
//
// dw and db: every workgroup writes the sums over its rows, a second kernel
// adds these partial sums in a fixed order, so results do not vary between
// runs.
#include "internal.h"
#include "lanes.h"

#include <algorithm>

namespace soap {
namespace {

// Workgroups of a launch at most.  Forward 1024 are four for every compute unit, more than
// are resident at once where a thread holds 32 values (144 registers and more: 768), whose
// last ones then start late: passes over changing inputs, 16384 x 4096 bfloat16 51.2 us (54
// with 768), but 16384 x 2048 26.8 (24.9), x 2047 43.6 (36.1), 8192 x 8192 53.8 (47.5).
// Backward they are the rows of partial sums: two for every compute unit where more than
// one fits it (16384 x 4096 bfloat16 81.6 us; 256 workgroups 93, 768 86, 1024 95), one past
// 4096 columns (8192 x 8192 fp32 153 us against 162 with 512, 4096 x 16384 bfloat16 96
// against 110).
constexpr int64_t LN_BLOCKS_FWD = 1024;
int64_t ln_most_bwd(int64_t cols) { return cols <= 4096 ? 512 : 256; }
constexpr int LN_FIN = 1024;             // threads of the second kernel,
constexpr int LN_FIN_COLS = 32;          // 32 columns x 32 slices

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v4u_any __attribute__((ext_vector_type(4), aligned(2)));   // 16 bytes at any element
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));

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

// Values of a unit of 16 bytes.
template <typename T>
constexpr int ln_vec() { return 16 / (int)sizeof(T); }

// The unit at column col of a row, zeros past its end.
template <typename T>
__device__ __forceinline__ v4u ln_load(const T *row, int col, int cols) {
  if (col + ln_vec<T>() <= cols) return *reinterpret_cast<const v4u_any *>(row + col);
  v4u q = v4u(0u);
#pragma unroll
  for (int i = 0; i < ln_vec<T>(); ++i)
    if (col + i < cols) {
      if constexpr (sizeof(T) == 4) q[i] = __float_as_uint(row[col + i]);
      else q[i / 2] |= (uint32_t)row[col + i] << (16 * (i & 1));
    }
  return q;
}

template <typename T>
__device__ __forceinline__ float ln_value(const v4u &q, int i) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(q[i]);
  else return __uint_as_float((i & 1) ? q[i / 2] & 0xffff0000u : q[i / 2] << 16);
}

template <typename T>
__device__ __forceinline__ void ln_store(T *row, int col, int cols, const float *v) {
  v4u q;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = __float_as_uint(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      q[i] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * i]) |
             ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * i + 1]) << 16);
  }
  if (col + ln_vec<T>() <= cols) {
    *reinterpret_cast<v4u_any *>(row + col) = q;
    return;
  }
#pragma unroll
  for (int i = 0; i < ln_vec<T>(); ++i)
    if (col + i < cols) {
      if constexpr (sizeof(T) == 4) row[col + i] = v[i];
      else row[col + i] = (uint16_t)(q[i / 2] >> (16 * (i & 1)));
    }
}

template <int VEC>
__device__ __forceinline__ void ln_param(const float *p, int col, int cols, float dflt, float *v) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) v[i] = dflt;
  if (!p) return;
  if (col + VEC <= cols) {
#pragma unroll
    for (int i = 0; i < VEC; i += 4) {
      const v4f q = *reinterpret_cast<const v4f_any *>(p + col + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i + j] = q[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (col + i < cols) v[i] = p[col + i];
  }
}

template <int GROUP>
constexpr int ln_threads() { return GROUP < 256 ? 256 : GROUP; }
template <int GROUP>
constexpr int ln_lanes() { return GROUP < 64 ? GROUP : 64; }

// Columns that the 64 threads of a wave (or the GROUP < 64 of a row) hold.
template <int VEC, int GROUP, int U>
__device__ __forceinline__ int ln_count(int cols, int first_thread) {
  constexpr int L = ln_lanes<GROUP>();
  int n = 0;
#pragma unroll
  for (int u = 0; u < U; ++u) n += min(max(cols - (u * GROUP + first_thread) * VEC, 0), L * VEC);
  return n;
}

template <typename T, int GROUP, int V>
__global__ __launch_bounds__(ln_threads<GROUP>()) void layer_norm_fwd(LnParams p) {
  constexpr int VEC = ln_vec<T>(), NT = ln_threads<GROUP>(), ROWS = NT / GROUP, U = V / VEC;
  constexpr int L = ln_lanes<GROUP>(), W = GROUP / L;   // waves of a row
  __shared__ float2 red[2][NT / 64];
  const int lane = threadIdx.x % GROUP, g = threadIdx.x / GROUP;
  const int wave = W > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  const float inv = 1.f / (float)p.cols;
  const float mine = (float)ln_count<VEC, GROUP, U>(p.cols, wave * 64);
  float w[U][VEC], b[U][VEC];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int col = (u * GROUP + lane) * VEC;
    ln_param<VEC>(p.w, col, p.cols, 1.f, w[u]);
    ln_param<VEC>(p.b, col, p.cols, 0.f, b[u]);
  }
  const int64_t step = (int64_t)gridDim.x * ROWS;
  int64_t row = (int64_t)blockIdx.x * ROWS + g;
  v4u next[U];
  auto load = [&](int64_t r) {
    const T *x = static_cast<const T *>(p.x) + min(r, p.rows - 1) * p.ldx;
#pragma unroll
    for (int u = 0; u < U; ++u) next[u] = ln_load<T>(x, (u * GROUP + lane) * VEC, p.cols);
  };
  load(row);
  for (int k = 0; row - g < p.rows; row += step, k ^= 1) {
    float v[U][VEC];
    float s = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        v[u][i] = ln_value<T>(next[u], i);
        s += v[u][i];
      }
    load(row + step);
    s = lane_sum<L>(s);
    float mu = W > 1 ? s / mine : s * inv;              // of the wave's columns, or the row's
    if (W > 1 && mine == 0.f) mu = 0.f;
    float q = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if ((u * GROUP + lane) * VEC + i < p.cols) {
          const float d = v[u][i] - mu;
          q = fmaf(d, d, q);
        }
    q = lane_sum<L>(q);
    if constexpr (W > 1) {
      // sum over waves of (squares about their mean + count (their mean - mean)^2)
      if ((threadIdx.x & 63) == 0) red[k][wave] = make_float2(s, q);
      __syncthreads();
      float2 o[W];
      s = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        o[i] = red[k][i];
        s += o[i].x;
      }
      mu = s * inv;
      q = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float n = (float)ln_count<VEC, GROUP, U>(p.cols, 64 * i);
        const float d = n > 0.f ? o[i].x / n - mu : 0.f;
        q += o[i].y + n * d * d;
      }
    }
    const float r = 1.f / sqrtf(q * inv + p.eps);
    if (row >= p.rows) continue;
    T *y = static_cast<T *>(p.out) + row * p.ldo;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int col = (u * GROUP + lane) * VEC;
      if (col >= p.cols) continue;
      float o[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) o[i] = fmaf((v[u][i] - mu) * r, w[u][i], b[u][i]);
      ln_store<T>(y, col, p.cols, o);
    }
    if (lane == 0) {
      if (p.mean) p.mean[row] = mu;
      if (p.rstd) p.rstd[row] = r;
    }
  }
}

// out = dx (none if null); part = the sums of dy h and dy over the workgroup's
// rows (none if null).
template <typename T, int GROUP, int V>
__global__ __launch_bounds__(ln_threads<GROUP>()) void layer_norm_bwd(LnParams p) {
  constexpr int VEC = ln_vec<T>(), NT = ln_threads<GROUP>(), ROWS = NT / GROUP, U = V / VEC;
  constexpr int L = ln_lanes<GROUP>(), W = GROUP / L;
  __shared__ float2 red[2][NT / 64];
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
  int64_t row = (int64_t)blockIdx.x * ROWS + g;
  v4u nx[U], nd[U];
  float nmu, nr;
  auto load = [&](int64_t r) {
    const int64_t at = min(r, p.rows - 1);
    const T *x = static_cast<const T *>(p.x) + at * p.ldx, *dy = static_cast<const T *>(p.dy) + at * p.lddy;
    nmu = p.mean_in[at];
    nr = p.rstd_in[at];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      nx[u] = ln_load<T>(x, (u * GROUP + lane) * VEC, p.cols);
      nd[u] = ln_load<T>(dy, (u * GROUP + lane) * VEC, p.cols);
    }
  };
  // Past 8192 columns the next row does not fit the registers, and the present one does not
  // quite: a thread keeps 20 (bfloat16) or 32 (fp32) of them in memory.  4096 x 16384
  // bfloat16 98 us, 4.1 TB/s, fp32 175, 4.6.
  constexpr bool AHEAD = GROUP < 512;
  if (AHEAD) load(row);
  for (int k = 0; row - g < p.rows; row += step, k ^= 1) {
    if (!AHEAD) load(row);
    const bool live = row < p.rows;
    const float mu = nmu, r = nr;
    float h[U][VEC], d[U][VEC];
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const bool in = live && (u * GROUP + lane) * VEC + i < p.cols;
        h[u][i] = in ? (ln_value<T>(nx[u], i) - mu) * r : 0.f;
        d[u][i] = in ? ln_value<T>(nd[u], i) : 0.f;
      }
    if (AHEAD) load(row + step);
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
    s1 = lane_sum<L>(s1);
    s2 = lane_sum<L>(s2);
    if constexpr (W > 1) {
      if ((threadIdx.x & 63) == 0) red[k][threadIdx.x >> 6] = make_float2(s1, s2);
      __syncthreads();
      s1 = s2 = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        s1 += red[k][i].x;
        s2 += red[k][i].y;
      }
    }
    if (!live) continue;
    s1 *= inv;
    s2 *= inv;
    T *dx = static_cast<T *>(p.out) + row * p.ldo;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int col = (u * GROUP + lane) * VEC;
      if (col >= p.cols) continue;
      float o[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) o[i] = r * (d[u][i] - s1 - h[u][i] * s2);
      ln_store<T>(dx, col, p.cols, o);
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
    for (int u = 0; u < U; ++u) {
      const int c = (u * GROUP + lane) * VEC;
#pragma unroll
      for (int i = 0; i < VEC; i += 4) {
        if (c + i + 4 <= p.cols) {
          *reinterpret_cast<v4f_any *>(part + c + i) = v4f{dw[u][i], dw[u][i + 1], dw[u][i + 2], dw[u][i + 3]};
          *reinterpret_cast<v4f_any *>(part + p.cols + c + i) =
              v4f{db[u][i], db[u][i + 1], db[u][i + 2], db[u][i + 3]};
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (c + i + j < p.cols) {
              part[c + i + j] = dw[u][i + j];
              part[p.cols + c + i + j] = db[u][i + j];
            }
        }
      }
    }
  }
}

// dw[c] or db[c] (by blockIdx.y) = sum over the workgroups' partial sums: slice s of
// 32 adds workgroups s, s + 32, ... in order, then the slices in order.
__global__ __launch_bounds__(LN_FIN) void layer_norm_bwd_finish(const float *__restrict__ part,
                                                               int nb, int cols,
                                                               float *__restrict__ dw,
                                                               float *__restrict__ db) {
  constexpr int C = LN_FIN_COLS, S = LN_FIN / C;
  __shared__ float red[LN_FIN];
  float *out = blockIdx.y == 0 ? dw : db;
  if (!out) return;
  const int c = blockIdx.x * C + threadIdx.x % C, s = threadIdx.x / C;
  float v = 0.f;
  if (c < cols) {
    const float *src = part + (int64_t)blockIdx.y * cols + c;
#pragma unroll 8
    for (int k = s; k < nb; k += S) v += src[(int64_t)k * 2 * cols];
  }
  red[threadIdx.x] = v;
  __syncthreads();
  if (s != 0 || c >= cols) return;
#pragma unroll
  for (int k = 1; k < S; ++k) v += red[k * C + threadIdx.x];
  out[c] = v;
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

int64_t ln_passes(int64_t rows, int64_t cols) {         // workgroups that would take one step each
  const int group = ln_shape(cols).group;
  const int64_t per = group < 256 ? 256 / group : 1;
  return (rows + per - 1) / per;
}
int64_t ln_blocks_fwd(int64_t rows, int64_t cols) { return std::min(ln_passes(rows, cols), LN_BLOCKS_FWD); }
// Backward, with few steps, as many workgroups as take the same number of them: no
// later, and fewer partial sums (1101 x 2303 fp32 17.8 us against 19.4 with 512; with
// many steps 512 is better, 30 000 x 1000 fp32 63.3 against 64.4).
int64_t ln_blocks_bwd(int64_t rows, int64_t cols) {
  const int64_t passes = ln_passes(rows, cols), most = ln_most_bwd(cols);
  if (passes > 4 * most) return most;
  const int64_t each = std::max<int64_t>(1, (passes + most - 1) / most);
  return (passes + each - 1) / each;
}

template <bool BWD, typename T>
hipError_t ln_launch(const LnParams &p, hipStream_t s) {
  const LnShape sh = ln_shape(p.cols);
  const dim3 grid((unsigned)BWD ? ln_blocks_bwd(p.rows, p.cols) : ln_blocks_fwd(p.rows, p.cols));
#define SOAP_LN(G, N)                                                                        \
  if (sh.group == G && sh.v == N) {                                                          \
    if constexpr (BWD)                                                                       \
      hipLaunchKernelGGL((layer_norm_bwd<T, G, N>), grid, dim3(ln_threads<G>()), 0, s, p);   \
    else                                                                                     \
      hipLaunchKernelGGL((layer_norm_fwd<T, G, N>), grid, dim3(ln_threads<G>()), 0, s, p);   \
    return hipGetLastError();                                                                \
  }
  SOAP_LN(8, 8) SOAP_LN(8, 16) SOAP_LN(8, 32)
  SOAP_LN(64, 8) SOAP_LN(64, 16) SOAP_LN(64, 32)
  SOAP_LN(256, 16) SOAP_LN(256, 32) SOAP_LN(512, 32)
#undef SOAP_LN
  return hipErrorInvalidValue;
}

}  // namespace

// At least what ln_blocks_bwd workgroups write, and growing with both arguments, so that a
// workspace of the largest call is enough for the others: even shares can take fewer
// workgroups for more rows, and rows past 4096 columns take half as many.
size_t layer_norm_part_bytes(int64_t rows, int64_t cols) {
  const int64_t passes = ln_passes(rows, cols), narrow = std::min<int64_t>(cols, 4096);
  const int64_t values = std::max(cols * std::min(passes, ln_most_bwd(cols)),
                                  narrow * std::min(passes, ln_most_bwd(narrow)));
  return sizeof(float) * 2 * values;
}

hipError_t launch_layer_norm_fwd(const LayerNormDesc &d, hipStream_t s) {
  if (d.rows <= 0) return hipSuccess;
  LnParams p{};
  p.rows = d.rows; p.cols = (int)d.cols;
  p.x = d.x; p.ldx = d.ldx; p.w = d.weight; p.b = d.bias; p.eps = d.eps;
  p.out = d.out; p.ldo = d.ldo; p.mean = d.mean; p.rstd = d.rstd;
  return d.bf16 ? ln_launch<false, uint16_t>(p, s) : ln_launch<false, float>(p, s);
}

hipError_t launch_layer_norm_bwd(const LayerNormDesc &d, hipStream_t s) {
  LnParams p{};
  p.rows = d.rows; p.cols = (int)d.cols;
  p.x = d.x; p.ldx = d.ldx; p.dy = d.dy; p.lddy = d.lddy; p.w = d.weight;
  p.mean_in = d.mean; p.rstd_in = d.rstd; p.out = d.out; p.ldo = d.ldo;
  const bool sums = d.dweight || d.dbias;      // without rows they are zeros, from no partial sums
  p.part = sums ? d.part : nullptr;
  hipError_t e = hipSuccess;
  if (d.rows > 0)
    e = d.bf16 ? ln_launch<true, uint16_t>(p, s) : ln_launch<true, float>(p, s);
  if (e != hipSuccess || !sums) return e;
  hipLaunchKernelGGL(layer_norm_bwd_finish, dim3((unsigned)((d.cols + LN_FIN_COLS - 1) / LN_FIN_COLS), 2), dim3(LN_FIN),
                     0, s, p.part, (int)ln_blocks_bwd(d.rows, d.cols), p.cols, d.dweight,
                     d.dbias);
  return hipGetLastError();
}

}  // namespace soap
