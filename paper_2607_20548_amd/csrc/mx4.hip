// Microscaled 4-bit floating point (MXFP4): blocks of 32 values along the summed
// axis share a power of two 2^e and hold x / 2^e as 4-bit values (sign, two bits
// of exponent, one of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6).
//
//   e = max(floor(log2 max|x|) - 2, -127), kept as the byte e + 127 (255 where the
//   block holds an infinity or a NaN: all its values stand for NaN); x / 2^e is
//   rounded to nearest, ties to even, and saturates at 6.
//
// With E the exponent field of max|x|, the byte is max(E - 2, 0), and 255 for
// E = 255: infinities and NaNs are found by comparing the bits of |x| as integers.
#include "internal.h"

#include <algorithm>

namespace soap {
namespace {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v8i __attribute__((ext_vector_type(8)));

// --------------------------------------------------------- quantisation
__device__ __forceinline__ uint32_t mx_abs(float f) { return __float_as_uint(f) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t mx_byte(uint32_t amax) {
  const uint32_t e = amax >> 23;
  return e == 255u ? 255u : e > 2u ? e - 2u : 0u;
}
__device__ __forceinline__ float mx_scale(uint32_t byte) {
  return __uint_as_float(byte ? byte << 23 : 0x400000u);   // 2^-127 is subnormal
}
// Maximum over aligned groups of 8 lanes.
__device__ __forceinline__ uint32_t mx_max8(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));    // lane ^ 1
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));    // lane ^ 2
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));  // 7 - lane
}

struct QuantParams {
  int64_t rows, cols, ldx, x_rows, sx;
  const void *x;
  const int *row_index;
  uint8_t *data, *scale, *data_t, *scale_t;
  int64_t kp, rp;          // padded columns and rows
  int vec;
};

// A workgroup takes 128 rows x 256 columns, a wave 32 rows of them and a lane
// four columns: every value is read once and both directions are formed in
// registers.  A block along the columns is eight lanes of one row, a block along
// the rows one column of a lane.
template <typename T, bool ROWS, bool COLS>
__global__ __launch_bounds__(256) void mx4_quantize(QuantParams p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t b = blockIdx.y;
  const int64_t ct = p.kp / 256, rt = blockIdx.x / ct;
  const int64_t r0 = (rt * 4 + wave) * 32;
  const int64_t c0 = (blockIdx.x - rt * ct) * 256 + 4 * lane;
  const T *x = static_cast<const T *>(p.x) + b * p.sx;
  if (r0 >= (COLS ? p.rp : p.rows)) return;
  float v[32][4];
  const bool in4 = c0 + 3 < p.cols;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const int64_t r = r0 + i;
    int64_t src = -1;
    if (r < p.rows) src = p.row_index ? (int64_t)p.row_index[r] : r;
    if (src >= p.x_rows) src = -1;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[i][j] = 0.f;
    if (src < 0) continue;
    const T *xr = x + src * p.ldx + c0;
    if (p.vec && in4) {
      if constexpr (sizeof(T) == 4) {
        const float4 q = *reinterpret_cast<const float4 *>(xr);
        v[i][0] = q.x; v[i][1] = q.y; v[i][2] = q.z; v[i][3] = q.w;
      } else {
        const uint2 q = *reinterpret_cast<const uint2 *>(xr);
        v[i][0] = __uint_as_float(q.x << 16); v[i][1] = __uint_as_float(q.x & 0xffff0000u);
        v[i][2] = __uint_as_float(q.y << 16); v[i][3] = __uint_as_float(q.y & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c0 + j < p.cols) {
          if constexpr (sizeof(T) == 4) v[i][j] = xr[j];
          else v[i][j] = __uint_as_float((uint32_t)xr[j] << 16);
        }
    }
  }
  if constexpr (ROWS) {
    uint8_t *data = p.data + b * p.rows * (p.kp / 2), *scale = p.scale + b * p.rows * (p.kp / 32);
    uint32_t keep[4];          // the byte of row 8 i + lane % 8 of the lane's block
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const uint32_t a = max(max(mx_abs(v[i][0]), mx_abs(v[i][1])), max(mx_abs(v[i][2]), mx_abs(v[i][3])));
      const uint32_t byte = mx_byte(mx_max8(a));
      const float s = mx_scale(byte);
      uint32_t q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[i][0], v[i][1], s, 0);
      q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[i][2], v[i][3], s, 1);
      const uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)q, 0xB1, 0xF, 0xF, true);
      if (r0 + i < p.rows && (lane & 1) == 0)
        *reinterpret_cast<uint32_t *>(data + (r0 + i) * (p.kp / 2) + c0 / 2) = q | (other << 16);
      if ((i & 7) == (lane & 7)) keep[i >> 3] = byte;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t r = r0 + 8 * i + (lane & 7);
      if (r < p.rows) scale[r * (p.kp / 32) + c0 / 32] = (uint8_t)keep[i];
    }
  }
  if constexpr (COLS) {
    uint8_t *data = p.data_t + b * p.cols * (p.rp / 2), *scale = p.scale_t + b * p.cols * (p.rp / 32);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t a = 0u;
#pragma unroll
      for (int i = 0; i < 32; ++i) a = max(a, mx_abs(v[i][j]));
      const uint32_t byte = mx_byte(a);
      const float s = mx_scale(byte);
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        w[k] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[8 * k][j], v[8 * k + 1][j], s, 0);
        w[k] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[k], v[8 * k + 2][j], v[8 * k + 3][j], s, 1);
        w[k] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[k], v[8 * k + 4][j], v[8 * k + 5][j], s, 2);
        w[k] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[k], v[8 * k + 6][j], v[8 * k + 7][j], s, 3);
      }
      if (c0 + j < p.cols) {
        *reinterpret_cast<uint4 *>(data + (c0 + j) * (p.rp / 2) + r0 / 2) = make_uint4(w[0], w[1], w[2], w[3]);
        scale[(c0 + j) * (p.rp / 32) + r0 / 32] = (uint8_t)byte;
      }
    }
  }
}

// The values of a packed matrix: eight per thread.
template <typename T>
__global__ __launch_bounds__(256) void mx4_dequantize(Mx4Mat a, int64_t rows, int64_t cols, int64_t kp,
                                                      T *__restrict__ out, int64_t ldo, int vec) {
  const int64_t per = (cols + 7) / 8, n = rows * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per, c = 8 * (i - r * per);
    const uint32_t q = *reinterpret_cast<const uint32_t *>(a.data + r * (kp / 2) + c / 2);
    const uint32_t byte = a.scale[r * (kp / 32) + c / 32];
    const float s = byte == 255u ? __uint_as_float(0x7fc00000u) : mx_scale(byte);
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t m = (q >> (4 * j)) & 7u;
      float f = m < 2u ? 0.5f * (float)m : __uint_as_float(((126u + (m >> 1)) << 23) | ((m & 1u) << 22));
      v[j] = ((q >> (4 * j)) & 8u ? -f : f) * s;
    }
    T *o = out + r * ldo + c;
    if (vec && c + 8 <= cols) {
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(o) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4 *>(o + 4) = make_float4(v[4], v[5], v[6], v[7]);
      } else {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[j] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * j]) |
                 ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * j + 1]) << 16);
        *reinterpret_cast<uint4 *>(o) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j < cols) {
          if constexpr (sizeof(T) == 4) o[j] = v[j];
          else o[j] = __builtin_bit_cast(uint16_t, (__bf16)v[j]);
        }
    }
  }
}

// -------------------------------------------------------------- products
struct MxParams {
  int64_t M, N, ldc, sC;      // M: rows of A (all groups together where rows are grouped)
  int kb;                     // blocks of 32 of a packed row that hold values
  int64_t bytes;              // data bytes of a packed row (16 a block); scales: bytes / 16
  int groups, tiles_n;
  const int *offsets;
  const uint8_t *A, *As, *B, *Bs;
  void *C;
};

enum { MX_ONE = 0, MX_ROWS = 1, MX_K = 2 };

// A tile's part of the problem: rows [m0, m1) of A and C, B's first row, blocks
// [kb0, kb1), C's first element.  Offsets are clamped into the matrix.
struct MxTile {
  int64_t m0, m1, b0, c0;
  int kb0, kb1;
};

// Tile t of BM rows among the groups' tiles (each group's rows start a tile of
// their own, the rows past the last group are a group of zeros).  Every wave
// finds it by itself: 64 groups at a time, an inclusive scan of their tiles.
template <int BM>
__device__ __forceinline__ bool mx_find(const MxParams &p, int64_t t, MxTile &o) {
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  for (int g0 = 0; g0 <= p.groups; g0 += 64) {
    const int g = g0 + lane;
    int64_t lo = 0, hi = 0;
    if (g <= p.groups) {
      lo = min(max((int64_t)p.offsets[g], (int64_t)0), p.M);
      hi = g < p.groups ? min(max((int64_t)p.offsets[g + 1], lo), p.M) : p.M;
    }
    int n = (int)((hi - lo + BM - 1) / BM), sum = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int u = __shfl_up(sum, d);
      if (lane >= d) sum += u;
    }
    const uint64_t past = __ballot(t < before + sum);
    if (past) {
      const int w = (int)__ffsll((unsigned long long)past) - 1;
      const int first = __shfl(sum - n, w);
      const int64_t glo = __shfl((int)lo, w), ghi = __shfl((int)hi, w);
      o.m0 = glo + (t - before - first) * BM;
      o.m1 = ghi;
      o.b0 = (int64_t)min(g0 + w, p.groups - 1) * p.N;
      o.c0 = 0;
      o.kb0 = 0;
      o.kb1 = g0 + w < p.groups ? p.kb : 0;
      return true;
    }
    before += __shfl(sum, 63);
  }
  return false;
}

template <int MODE, int BM>
__device__ __forceinline__ bool mx_tile(const MxParams &p, int64_t t, MxTile &o) {
  if constexpr (MODE == MX_ROWS) return mx_find<BM>(p, t, o);
  o.m0 = t * BM; o.m1 = p.M; o.b0 = 0; o.c0 = 0; o.kb0 = 0; o.kb1 = p.kb;
  if constexpr (MODE == MX_K) {
    const int g = blockIdx.y;
    o.kb0 = min(max(p.offsets[g] >> 5, 0), p.kb);
    o.kb1 = min(max(p.offsets[g + 1] >> 5, o.kb0), p.kb);
    o.c0 = g * p.sC;
  }
  return true;
}

template <typename T>
__device__ __forceinline__ void mx_put(T *c, float v) {
  if constexpr (sizeof(T) == 4) *c = v;
  else *c = __builtin_bit_cast(uint16_t, (__bf16)v);
}

// 32 x 128 of C per workgroup, 32 x 32 per wave, operands straight from memory:
// a lane of a matrix instruction takes a whole block (16 bytes) and its scale.
template <int MODE, typename T>
__global__ __launch_bounds__(256) void mx4_gemm(MxParams p) {
  MxTile o;
  const int64_t tm = blockIdx.x / p.tiles_n, tn = blockIdx.x - tm * p.tiles_n;
  if (!mx_tile<MODE, 32>(p, tm, o)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, xl = lane & 31, h = lane >> 5;
  const int64_t n0 = tn * 128 + 32 * wave;
  if (o.m0 >= o.m1 || n0 >= p.N) return;
  const int64_t ra = min(o.m0 + xl, o.m1 - 1), rb = o.b0 + min(n0 + xl, p.N - 1);
  const uint8_t *a = p.A + ra * p.bytes, *b = p.B + rb * p.bytes;
  const uint8_t *as = p.As + ra * (p.bytes / 16), *bs = p.Bs + rb * (p.bytes / 16);
  v16f acc;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0.f;
  for (int k = o.kb0; k < o.kb1; k += 2) {
    const bool live = k + h < o.kb1;
    const int kk = live ? k + h : k;
    uint4 x = *reinterpret_cast<const uint4 *>(a + 16 * (int64_t)kk);
    uint4 y = *reinterpret_cast<const uint4 *>(b + 16 * (int64_t)kk);
    int sx = as[kk], sy = bs[kk];
    if (!live) {
      x = y = make_uint4(0u, 0u, 0u, 0u);
      sx = sy = 127;
    }
    const v8i va = {(int)x.x, (int)x.y, (int)x.z, (int)x.w, 0, 0, 0, 0};
    const v8i vb = {(int)y.x, (int)y.y, (int)y.z, (int)y.w, 0, 0, 0, 0};
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(va, vb, acc, 4, 4, 0, sx, 0, sy);
  }
  T *C = static_cast<T *>(p.C) + o.c0;
  if (n0 + xl >= p.N) return;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int64_t row = o.m0 + 8 * (r >> 2) + 4 * h + (r & 3);
    if (row < o.m1) mx_put<T>(C + row * p.ldc + n0 + xl, acc[r]);
  }
}

template <int MODE, typename T>
hipError_t mx_launch(MxParams p, hipStream_t s) {
  const int64_t tm = (p.M + 31) / 32 + (MODE == MX_ROWS ? p.groups + 1 : 0);
  p.tiles_n = (int)((p.N + 127) / 128);
  if (tm * p.tiles_n > INT32_MAX) return hipErrorInvalidValue;
  hipLaunchKernelGGL((mx4_gemm<MODE, T>),
                     dim3((unsigned)(tm * p.tiles_n), MODE == MX_K ? p.groups : 1), dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_quantize(const Mx4QuantDesc &d, hipStream_t s) {
  if (d.batch <= 0 || d.cols <= 0) return hipSuccess;
  QuantParams p{};
  p.rows = d.rows; p.cols = d.cols; p.ldx = d.ldx; p.x_rows = d.x_rows; p.sx = d.rows * d.ldx;
  p.x = d.x; p.row_index = d.row_index;
  p.data = d.data; p.scale = d.scale; p.data_t = d.data_t; p.scale_t = d.scale_t;
  p.kp = mx4_padded(d.cols); p.rp = mx4_padded(d.rows);
  const int need = d.bf16 ? 8 : 16, elem = d.bf16 ? 2 : 4;
  p.vec = reinterpret_cast<uintptr_t>(d.x) % need == 0 && d.ldx * elem % need == 0;
  const bool cols = d.data_t != nullptr, rows = d.data != nullptr;
  const int64_t rt = ((cols ? p.rp : d.rows) + 127) / 128, ct = p.kp / 256;
  if (rt == 0) return hipSuccess;
  if (ct * rt > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(ct * rt), (unsigned)d.batch);
#define SOAP_MXQ(T, R, C) hipLaunchKernelGGL((mx4_quantize<T, R, C>), grid, dim3(256), 0, s, p)
  if (d.bf16) {
    if (rows && cols) SOAP_MXQ(uint16_t, true, true);
    else if (rows) SOAP_MXQ(uint16_t, true, false);
    else SOAP_MXQ(uint16_t, false, true);
  } else {
    if (rows && cols) SOAP_MXQ(float, true, true);
    else if (rows) SOAP_MXQ(float, true, false);
    else SOAP_MXQ(float, false, true);
  }
#undef SOAP_MXQ
  return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const Mx4Mat &a, int64_t rows, int64_t cols, bool bf16, void *out,
                                 int64_t ldo, hipStream_t s) {
  if (rows <= 0) return hipSuccess;
  const int64_t n = rows * ((cols + 7) / 8);
  const dim3 grid((unsigned)std::min<int64_t>((n + 255) / 256, 16384));
  const bool vec = (reinterpret_cast<uintptr_t>(out) & 15u) == 0 && ldo * (bf16 ? 2 : 4) % 16 == 0;
  if (bf16)
    hipLaunchKernelGGL((mx4_dequantize<uint16_t>), grid, dim3(256), 0, s, a, rows, cols, mx4_padded(cols),
                       static_cast<uint16_t *>(out), ldo, (int)vec);
  else
    hipLaunchKernelGGL((mx4_dequantize<float>), grid, dim3(256), 0, s, a, rows, cols, mx4_padded(cols),
                       static_cast<float *>(out), ldo, (int)vec);
  return hipGetLastError();
}

hipError_t launch_mx4_gemm(const Mx4GemmDesc &d, hipStream_t s) {
  if (d.M <= 0 || d.N <= 0 || d.groups <= 0) return hipSuccess;
  MxParams p{};
  p.M = d.M; p.N = d.N; p.ldc = d.ldc; p.sC = d.M * d.ldc;
  p.kb = (int)((d.K + 31) / 32); p.bytes = mx4_padded(d.K) / 2;
  p.groups = (int)d.groups; p.offsets = d.offsets;
  p.A = d.A.data; p.As = d.A.scale; p.B = d.B.data; p.Bs = d.B.scale; p.C = d.C;
  const int mode = !d.offsets ? MX_ONE : d.by_k ? MX_K : MX_ROWS;
#define SOAP_MXG(T)                                   \
  (mode == MX_ONE ? mx_launch<MX_ONE, T>(p, s)        \
   : mode == MX_ROWS ? mx_launch<MX_ROWS, T>(p, s)    \
                     : mx_launch<MX_K, T>(p, s))
  return d.bf16 ? SOAP_MXG(uint16_t) : SOAP_MXG(float);
#undef SOAP_MXG
}

}  // namespace soap
