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
#include <type_traits>

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
  int groups, tiles_m, tiles_n;
  int wide;                   // C can be written 16 bytes at a time
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
      const int first = __builtin_amdgcn_readlane(sum - n, w);
      const int64_t glo = __builtin_amdgcn_readlane((int)lo, w), ghi = __builtin_amdgcn_readlane((int)hi, w);
      o.m0 = glo + (t - before - first) * BM;
      o.m1 = ghi;
      o.b0 = (int64_t)min(g0 + w, p.groups - 1) * p.N;
      o.c0 = 0;
      o.kb0 = 0;
      o.kb1 = g0 + w < p.groups ? p.kb : 0;
      return true;
    }
    before += __builtin_amdgcn_readlane(sum, 63);
  }
  return false;
}

template <int MODE, int BM>
__device__ __forceinline__ bool mx_tile(const MxParams &p, int64_t t, int g, MxTile &o) {
  if constexpr (MODE == MX_ROWS) return mx_find<BM>(p, t, o);
  o.m0 = t * BM; o.m1 = p.M; o.b0 = 0; o.c0 = 0; o.kb0 = 0; o.kb1 = p.kb;
  if constexpr (MODE == MX_K) {
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
  if (!mx_tile<MODE, 32>(p, tm, blockIdx.y, o)) return;
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

// The same product by tiles of TM x TN through LDS: four waves (2 x 2), each
// (TM / 2) x (TN / 2) in blocks of 32 x 32.  K advances in slabs of 256 values (128
// bytes of a row, eight blocks), two in LDS, written there by the loads
// themselves (16 bytes a lane, no registers): unit g of row x lies at position
// g ^ (x / 2 % 8) of its 128 bytes, so that sixteen consecutive rows of one unit
// are in different banks, and each lane fetches the unit that its place in LDS
// wants.  The scales come 16 bytes a row, two slabs' worth, likewise.  A matrix
// instruction takes 64 values: lane (row, h) block 2 q + h of the slab at step q,
// the scale being byte q of the row's even or odd scales.
//
// One barrier a slab: before the last of its four steps, whose fragments are read
// by then, it makes the next slab visible and this one free, the loads of the
// slab after the next start there, and the last step reads the next slab's first
// fragments, each step multiplying what was read during the one before.
//
// Slabs are whole in the packed rows; blocks outside [kb0, kb1), the neighbours'
// or padding, are multiplied as zeros.  The B operand goes first, so that a lane
// holds four consecutive columns of one row of C: results are rounded in
// registers, staged 32 rows at a time in the wave's part of the LDS and written
// 16 bytes a lane.
__device__ __forceinline__ void mx_dma16(uint32_t lds, const uint8_t *base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
// All of the workgroup's loads into LDS have landed, and its LDS reads are done.
__device__ __forceinline__ void mx_sync() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

template <int TM, int TN>
struct MxLds {
  static constexpr int ROWS = TM + TN;             // A's rows, then B's
  static constexpr int DATA = ROWS * 128, SCALE = ROWS * 16;
  static constexpr int BYTES = 2 * (DATA + SCALE);
};

template <int MODE, typename T, int TM, int TN>
__global__ __launch_bounds__(256, TM == 256 ? 1 : 2) void mx4_gemm_tile(MxParams p) {
  typedef MxLds<TM, TN> L;
  constexpr int BI = TM / 64, BJ = TN / 64;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[L::BYTES];
  const int nt = gridDim.x;
  int t = blockIdx.x;
  {                                       // a contiguous run of tiles per XCD
    const int x = t & 7, per = nt >> 3, more = nt & 7;
    t = x * per + min(x, more) + (t >> 3);
  }
  int g = 0;
  if constexpr (MODE == MX_K) {
    g = t / (p.tiles_m * p.tiles_n);
    t -= g * p.tiles_m * p.tiles_n;
  }
  // eight tiles of rows by all tiles of columns at a time
  const int per_group = 8 * p.tiles_n, group = t / per_group, first = group * 8;
  const int gsz = min(p.tiles_m - first, 8), in_group = t - group * per_group;
  const int tm = first + in_group % gsz, tn = in_group / gsz;
  MxTile o;
  if (!mx_tile<MODE, TM>(p, tm, g, o)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 1, wn = wave & 1;
  const int xl = lane & 31, h = lane >> 5;
  const int64_t m0 = o.m0, n0 = (int64_t)tn * TN;
  if (m0 >= o.m1) return;

  v16f acc[BI][BJ];
#pragma unroll
  for (int i = 0; i < BI; ++i)
#pragma unroll
    for (int j = 0; j < BJ; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
  const int am = (int)min((int64_t)TM, o.m1 - m0) - 1, bm = (int)min((int64_t)TN, p.N - n0) - 1;
  const uint8_t *abase = p.A + m0 * p.bytes, *bbase = p.B + (o.b0 + n0) * p.bytes;
  const int64_t srow = p.bytes / 16;
  const uint8_t *asbase = p.As + m0 * srow, *bsbase = p.Bs + (o.b0 + n0) * srow;
  // data: load s of a wave brings rows 32 s + 8 wave .. + 7
  uint32_t aoff[TM / 32], boff[TN / 32];
  const int lr = 8 * wave + (lane >> 3), unit = (lane & 7) ^ ((lr >> 1) & 7);
#pragma unroll
  for (int s = 0; s < TM / 32; ++s) aoff[s] = (uint32_t)(min(32 * s + lr, am) * p.bytes + 16 * unit);
#pragma unroll
  for (int s = 0; s < TN / 32; ++s) boff[s] = (uint32_t)(min(32 * s + lr, bm) * p.bytes + 16 * unit);
  // scales: load s of a wave brings rows 64 (4 s + wave) .. + 63 of A's and B's
  constexpr int SL = L::ROWS / 256;
  uint32_t soff[SL];
#pragma unroll
  for (int s = 0; s < SL; ++s) {
    const int r = 64 * (4 * s + wave);
    soff[s] = (uint32_t)((r < TM ? min(r + lane, am) : min(r - TM + lane, bm)) * srow);
  }
  const int slabs = (int)(p.bytes >> 7);           // of a packed row; at least 2
  const int s0 = o.kb0 >> 3, s1 = o.kb1 > o.kb0 ? (o.kb1 + 7) >> 3 : s0;
  auto load = [&](int s) {                         // slab s; past the last: nothing
    if (s >= s1) return;
    const uint32_t dst = lds0 + (s & 1) * L::DATA + wave * 1024;
    const uint8_t *a = abase + 128 * (int64_t)s, *b = bbase + 128 * (int64_t)s;
#pragma unroll
    for (int i = 0; i < TM / 32; ++i) mx_dma16(dst + i * 4096, a, aoff[i]);
#pragma unroll
    for (int i = 0; i < TN / 32; ++i) mx_dma16(dst + TM * 128 + i * 4096, b, boff[i]);
    if ((s & 1) == 0 || s == s0) {
      const int at = 8 * min(s & ~1, slabs - 2);
#pragma unroll
      for (int i = 0; i < SL; ++i) {
        const int r = 64 * (4 * i + wave);
        mx_dma16(lds0 + 2 * L::DATA + ((s >> 1) & 1) * L::SCALE + r * 16, (r < TM ? asbase : bsbase) + at,
                 soff[i]);
      }
    }
  };

  uint4 fa[2][BI], fb[2][BJ];
  uint32_t sa[2][BI], sb[2][BJ];
  const int sw = (xl >> 1) & 7;
  const int arow = wm * (TM / 2) + xl, brow = TM + wn * (TN / 2) + xl;
  const uint32_t half = h ? 0x07050301u : 0x06040200u;
  auto frag = [&](int f, int s, int q) {
    const uint8_t *d = lds + (s & 1) * L::DATA + 16 * ((2 * q + h) ^ sw);
#pragma unroll
    for (int i = 0; i < BI; ++i) fa[f][i] = *reinterpret_cast<const uint4 *>(d + (arow + 32 * i) * 128);
#pragma unroll
    for (int j = 0; j < BJ; ++j) fb[f][j] = *reinterpret_cast<const uint4 *>(d + (brow + 32 * j) * 128);
  };
  auto scales = [&](int f, int s) {
    const uint8_t *d = lds + 2 * L::DATA + ((s >> 1) & 1) * L::SCALE + 8 * (s - min(s & ~1, slabs - 2));
#pragma unroll
    for (int i = 0; i < BI; ++i) {
      const uint2 v = *reinterpret_cast<const uint2 *>(d + (arow + 32 * i) * 16);
      sa[f][i] = __builtin_amdgcn_perm(v.y, v.x, half);
    }
#pragma unroll
    for (int j = 0; j < BJ; ++j) {
      const uint2 v = *reinterpret_cast<const uint2 *>(d + (brow + 32 * j) * 16);
      sb[f][j] = __builtin_amdgcn_perm(v.y, v.x, half);
    }
  };
  auto multiply = [&](auto step, int f, int fs, int s) {
    constexpr int q = decltype(step)::value;
    const int kb = 8 * s + 2 * q;
    if (kb < o.kb0 || kb + 2 > o.kb1) {            // a block of the two is not this product's
      const bool live = kb + h >= o.kb0 && kb + h < o.kb1;
#pragma unroll
      for (int i = 0; i < BI; ++i) {
        if (!live) fa[f][i] = make_uint4(0u, 0u, 0u, 0u);
        if (!live) sa[fs][i] = (sa[fs][i] & ~(0xffu << (8 * q))) | (127u << (8 * q));
      }
#pragma unroll
      for (int j = 0; j < BJ; ++j)
        if (!live) sb[fs][j] = (sb[fs][j] & ~(0xffu << (8 * q))) | (127u << (8 * q));
    }
#pragma unroll
    for (int i = 0; i < BI; ++i)
#pragma unroll
      for (int j = 0; j < BJ; ++j) {
        const uint4 x = fa[f][i], y = fb[f][j];
        const v8i va = {(int)x.x, (int)x.y, (int)x.z, (int)x.w, 0, 0, 0, 0};
        const v8i vb = {(int)y.x, (int)y.y, (int)y.z, (int)y.w, 0, 0, 0, 0};
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(vb, va, acc[i][j], 4, 4, q, (int)sb[fs][j],
                                                                    q, (int)sa[fs][i]);
      }
  };
  using std::integral_constant;
  if (s1 > s0) {
    load(s0);
    mx_sync();
    load(s0 + 1);
    frag(0, s0, 0);
    scales(0, s0);
    for (int s = s0; s < s1; ++s) {
      frag(1, s, 1);
      multiply(integral_constant<int, 0>{}, 0, 0, s);
      frag(0, s, 2);
      multiply(integral_constant<int, 1>{}, 1, 0, s);
      frag(1, s, 3);
      multiply(integral_constant<int, 2>{}, 0, 0, s);
      mx_sync();
      load(s + 2);
      const bool more = s + 1 < s1;
      if (more) {
        frag(0, s + 1, 0);
        scales(1, s + 1);
      }
      multiply(integral_constant<int, 3>{}, 1, 0, s);
      if (more) {
#pragma unroll
        for (int i = 0; i < BI; ++i) sa[0][i] = sa[1][i];
#pragma unroll
        for (int j = 0; j < BJ; ++j) sb[0][j] = sb[1][j];
      }
    }
  }

  // Register r of block (i, j) is C[32 i + xl][32 j + 8 (r / 4) + 4 h + r % 4].
  constexpr int WN = TN / 2, E = sizeof(T), STRIDE = WN * E + 16, PER = 16 / E;
  static_assert(4 * 32 * STRIDE <= L::BYTES, "the staged rows fit the LDS");
  uint8_t *stage = lds + wave * 32 * STRIDE;
  T *C = static_cast<T *>(p.C) + o.c0;
  const int64_t cw = n0 + wn * WN;
  mx_sync();
#pragma unroll
  for (int i = 0; i < BI; ++i) {
#pragma unroll
    for (int j = 0; j < BJ; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float v0 = acc[i][j][4 * r], v1 = acc[i][j][4 * r + 1], v2 = acc[i][j][4 * r + 2],
                    v3 = acc[i][j][4 * r + 3];
        uint8_t *d = stage + xl * STRIDE + (32 * j + 8 * r + 4 * h) * E;
        if constexpr (E == 4) {
          *reinterpret_cast<float4 *>(d) = make_float4(v0, v1, v2, v3);
        } else {
          const uint32_t lo = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v0) |
                              ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v1) << 16);
          const uint32_t hi = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v2) |
                              ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v3) << 16);
          *reinterpret_cast<uint2 *>(d) = make_uint2(lo, hi);
        }
      }
    __builtin_amdgcn_wave_barrier();
    constexpr int LANES = WN / PER, RPI = 64 / LANES;       // lanes of a row, rows of an access
    const int er = lane / LANES, ec = PER * (lane % LANES);
#pragma unroll
    for (int u = 0; u < 32 / RPI; ++u) {
      const int x = er + RPI * u;
      const int64_t row = m0 + wm * (TM / 2) + 32 * i + x, col = cw + ec;
      const uint4 v = *reinterpret_cast<const uint4 *>(stage + x * STRIDE + ec * E);
      if (row >= o.m1 || col >= p.N) continue;
      T *dst = C + row * p.ldc + col;
      if (p.wide && col + PER <= p.N) {
        *reinterpret_cast<uint4 *>(dst) = v;
      } else {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < PER; ++e)
          if (col + e < p.N) {
            if constexpr (E == 4) dst[e] = __uint_as_float(w[e]);
            else dst[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
          }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

template <int MODE, typename T, int TM, int TN>
hipError_t mx_launch_tile(MxParams p, hipStream_t s) {
  const int64_t tm = (p.M + TM - 1) / TM + (MODE == MX_ROWS ? p.groups + 1 : 0), tn = (p.N + TN - 1) / TN;
  const int64_t n = tm * tn * (MODE == MX_K ? p.groups : 1);
  if (n > INT32_MAX) return hipErrorInvalidValue;
  p.tiles_m = (int)tm;
  p.tiles_n = (int)tn;
  hipLaunchKernelGGL((mx4_gemm_tile<MODE, T, TM, TN>), dim3((unsigned)n), dim3(256), 0, s, p);
  return hipGetLastError();
}

// Tiles through LDS where a packed row has two slabs at least (a load of scales
// brings two) and the 32-bit offsets of a tile's rows reach it.  256 x 256 where
// they fill the compute units, one each: 4096 x 4096 x 14336 133 us against 155 in
// 128-tiles, 2048 x 2048 x 2048 22 against 12.5, 512 x 14336 x 4096 38 against 24.5.
// Grouped rows leave the last tile of each group part empty: 128-tiles (64 experts
// of 2048 x 768, 512 rows each, 54 us against 74).
template <int MODE, typename T>
hipError_t mx_launch(MxParams p, hipStream_t s) {
  if (p.bytes >= 256 && p.bytes <= (1 << 24)) {
    const int64_t n256 = (p.M + 255) / 256 * ((p.N + 255) / 256);
    if (MODE == MX_ONE && n256 >= 256) return mx_launch_tile<MODE, T, 256, 256>(p, s);
    return mx_launch_tile<MODE, T, 128, 128>(p, s);
  }
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
  const int64_t elem = d.bf16 ? 2 : 4;
  p.wide = (reinterpret_cast<uintptr_t>(d.C) & 15u) == 0 && d.ldc * elem % 16 == 0 &&
           (!d.by_k || p.sC * elem % 16 == 0);
  const int mode = !d.offsets ? MX_ONE : d.by_k ? MX_K : MX_ROWS;
#define SOAP_MXG(T)                                   \
  (mode == MX_ONE ? mx_launch<MX_ONE, T>(p, s)        \
   : mode == MX_ROWS ? mx_launch<MX_ROWS, T>(p, s)    \
                     : mx_launch<MX_K, T>(p, s))
  return d.bf16 ? SOAP_MXG(uint16_t) : SOAP_MXG(float);
#undef SOAP_MXG
}

}  // namespace soap
