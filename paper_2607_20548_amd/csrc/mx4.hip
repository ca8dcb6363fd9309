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
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint16_t v2h __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef uint32_t v4u_any __attribute__((ext_vector_type(4), aligned(2)));   // at any element
typedef uint32_t v2u_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t v8u __attribute__((ext_vector_type(8)));

// --------------------------------------------------------- quantisation
__device__ __forceinline__ uint32_t mx_byte(uint32_t e) { return e == 255u ? 255u : e > 2u ? e - 2u : 0u; }
__device__ __forceinline__ float mx_scale(uint32_t byte) {
  return __uint_as_float(byte ? byte << 23 : 0x400000u);   // 2^-127 is subnormal
}
// Two bfloat16 of a word: their maxima as integers, the low (high) halves of two words.
__device__ __forceinline__ uint32_t mx_max(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(v2h, a), __builtin_bit_cast(v2h, b)));
}
__device__ __forceinline__ uint32_t mx_low(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t mx_high(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
// Two values into byte SEL of q.  Both forms round alike (all bfloat16 at all scales compared).
template <int SEL>
__device__ __forceinline__ uint32_t mx_cvt(uint32_t q, uint32_t a, uint32_t b, float s) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(a), __uint_as_float(b), s, SEL);
}
template <int SEL>
__device__ __forceinline__ uint32_t mx_cvt(uint32_t q, uint32_t ab, float s) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(v2bf, ab), s, SEL);
}
// Maximum over aligned groups of 8 lanes, of a word or of its halves.
template <typename V>
__device__ __forceinline__ uint32_t mx_max8(uint32_t v) {
  auto most = [](uint32_t a, uint32_t b) {
    if constexpr (std::is_same<V, v2h>::value) return mx_max(a, b);
    else return max(a, b);
  };
  v = most(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));    // lane ^ 1
  v = most(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));    // lane ^ 2
  return most(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));  // 7 - lane
}

struct QuantParams {
  int64_t rows, cols, ldx, x_rows, sx;
  const void *x;
  const int *row_index;
  uint8_t *data, *scale, *data_t, *scale_t;
  int64_t kp, rp;          // padded columns and rows
};

// Along the columns only: eight values per lane, a block is four lanes of a row, so
// that a wave's loads and stores are contiguous.  A row has LPR lanes, which walk
// along it in QC_UNITS independent loads at a time; short rows have fewer lanes, so
// that all the loads are used (400 000 x 256 bfloat16 47 us with 16 lanes, 77 with 32;
// 131 072 x 768 44 with 32, 60 with 64; 16384 x 4096 34 with 32, 30 with 64).
constexpr int QC_UNITS = 4;
int mx_lanes(int64_t kp, int64_t most16, int64_t most32) { return kp <= most16 ? 16 : kp <= most32 ? 32 : 64; }
template <typename T, int LPR>
__global__ __launch_bounds__(256) void mx4_quantize_cols(QuantParams p) {
  constexpr int ROWS = 256 / LPR;
  const int64_t b = blockIdx.y;
  const T *x = static_cast<const T *>(p.x) + b * p.sx;
  uint8_t *data = p.data + b * p.rows * (p.kp / 2), *scale = p.scale + b * p.rows * (p.kp / 32);
  typedef typename std::conditional<sizeof(T) == 4, v8u, v4u>::type Raw;
  const int lane = threadIdx.x % LPR;
  for (int64_t r = (int64_t)blockIdx.x * ROWS + threadIdx.x / LPR; r < p.rows; r += (int64_t)gridDim.x * ROWS) {
    int64_t src = r;
    if (p.row_index) {
      src = p.row_index[r];
      if (src >= p.x_rows) src = -1;
    }
    const T *xr = x + src * p.ldx;
    uint8_t *dr = data + r * (p.kp / 2), *sr = scale + r * (p.kp / 32);
    for (int64_t c0 = 8 * lane; c0 < p.kp; c0 += QC_UNITS * LPR * 8) {
      Raw raw[QC_UNITS];
#pragma unroll
      for (int u = 0; u < QC_UNITS; ++u) {
        const int64_t c = c0 + u * LPR * 8;
        raw[u] = Raw(0u);
        if (src < 0 || c >= p.cols) continue;
        if (c + 8 <= p.cols) {
          if constexpr (sizeof(T) == 4) {
            const v4u lo = *reinterpret_cast<const v4u_any *>(xr + c), hi = *reinterpret_cast<const v4u_any *>(xr + c + 4);
            raw[u] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          } else {
            raw[u] = *reinterpret_cast<const v4u_any *>(xr + c);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (c + j < p.cols) {
              if constexpr (sizeof(T) == 4) raw[u][j] = __float_as_uint(xr[c + j]);
              else raw[u][j / 2] |= (uint32_t)xr[c + j] << (16 * (j & 1));
            }
        }
      }
#pragma unroll
      for (int u = 0; u < QC_UNITS; ++u) {
        const int64_t c = c0 + u * LPR * 8;
        auto bits = [&](int j) -> uint32_t {
          if constexpr (sizeof(T) == 4) return raw[u][j];
          else return (j & 1) ? raw[u][j / 2] & 0xffff0000u : raw[u][j / 2] << 16;
        };
        auto val = [&](int j) { return __uint_as_float(bits(j)); };
        uint32_t a = 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) a = max(a, bits(j) & 0x7fffffffu);
        a = max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0xB1, 0xF, 0xF, true));   // lane ^ 1
        a = max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0x4E, 0xF, 0xF, true));   // lane ^ 2
        const uint32_t byte = mx_byte(a >> 23);
        const float s = mx_scale(byte);
        uint32_t q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, val(0), val(1), s, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, val(2), val(3), s, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, val(4), val(5), s, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, val(6), val(7), s, 3);
        if (c < p.kp) {
          *reinterpret_cast<uint32_t *>(dr + c / 2) = q;
          if ((lane & 3) == 0) sr[c / 32] = (uint8_t)byte;
        }
      }
    }
  }
}

// Along the rows, or both ways: a workgroup takes 128 rows x 256 columns, a wave 32
// rows of them and a lane four columns: every value is read once and both
// directions are formed in registers.  A block along the columns is eight lanes of
// one row, a block along the rows one column of a lane; those go through LDS, so
// that a column's 64 bytes (four blocks) are written together.  Workgroups of
// consecutive rows run on one XCD, whose L2 joins what they write of a line.  Without
// an index no row is read twice: the loads leave the L2s to the stores (the 64 x 2048 x
// 768 bank both ways 90 us, 5.6 TB/s, against 103); with one, a token's row is read for
// each of its experts and kept there (34 752 rows of 4096 tokens of 2048 along the rows 18 us
// on one input, 20.6 in a kernel trace over changing ones).  The rows' loads do not wait for each other: a
// branch for every row or column that is not there took 65536 x 700 bfloat16 from 30 us
// to 79.  Bfloat16 maxima and conversions work on pairs, both ways 49 152 x 2048 60 us
// against 75 by single values (which held 256 registers, as fp32 does; with an index and both
// ways one fp32 value of a thread goes through memory).
template <typename T, bool ROWS, bool GATHER>
__global__ __launch_bounds__(256, 2) void mx4_quantize_tile(QuantParams p) {
  // column x's block of wave w: 16 bytes at x * 64 + 16 * (w ^ (x / 4 % 4))
  __shared__ __attribute__((aligned(16))) uint8_t lds[256 * 64 + 256 * 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t b = blockIdx.y;
  const int rt = (int)((p.rp + 127) / 128);
  int t;
  {
    const int nt = gridDim.x, x = blockIdx.x & 7, per = nt >> 3, more = nt & 7;
    t = x * per + min(x, more) + (int)(blockIdx.x >> 3);
  }
  const int64_t ct = __builtin_amdgcn_readfirstlane(t / rt), r0 = ((int64_t)(t - (int)ct * rt) * 4 + wave) * 32;
  const int64_t cw = ct * 256, c0 = cw + 4 * lane;
  const T *x = static_cast<const T *>(p.x) + b * p.sx;
  typedef typename std::conditional<sizeof(T) == 4, v4u, v2u>::type Raw;
  typedef typename std::conditional<sizeof(T) == 4, v4u_any, v2u_any>::type RawAny;
  // Lane i's row of x is row i's; bit i: there is one.
  int mine = 0;
  bool in = lane < 32 && r0 + lane < p.rows;
  if constexpr (GATHER) {
    if (in) mine = p.row_index[r0 + lane];
    in = in && mine >= 0 && mine < p.x_rows;
    if (!in) mine = 0;
  }
  const uint32_t ok = (uint32_t)__ballot(in);
  const int last = __builtin_amdgcn_readfirstlane((int)min(p.rows - r0, (int64_t)32) - 1);
  auto row = [&](int i) {
    return x + (GATHER ? (int64_t)__builtin_amdgcn_readlane(mine, i) : r0 + min(i, last)) * p.ldx;
  };
  // Whole loads of every row, rows without values row 0's, those at the right edge the
  // last four columns; what does not belong there goes out after all are on their way.
  Raw raw[32];
  if (ok == 0u || p.cols < 4) {
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      raw[i] = Raw(0u);
      if (!(ok >> i & 1u)) continue;
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (c0 + j < p.cols) {
          if constexpr (sizeof(T) == 4) raw[i][j] = __float_as_uint(row(i)[c0 + j]);
          else raw[i][j / 2] |= (uint32_t)row(i)[c0 + j] << (16 * (j & 1));
        }
    }
  } else {
    const int room = __builtin_amdgcn_readfirstlane((int)min(p.cols - cw, (int64_t)256));
    const int left = min(room - 4, 0), c = min(4 * lane, room - 4);
    const uint32_t at = (uint32_t)(c - left) * (uint32_t)sizeof(T);
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      uint64_t base = reinterpret_cast<uint64_t>(row(i) + cw + left);
      asm("" : "+s"(base));                    // the row's address stays a scalar, the lane's part an offset
      typedef const char __attribute__((address_space(1))) *Global;
      const auto from = reinterpret_cast<const RawAny __attribute__((address_space(1))) *>(reinterpret_cast<Global>(base) + at);
      if constexpr (GATHER) raw[i] = *from;
      else raw[i] = __builtin_nontemporal_load(from);
    }
    if (ok != ~0u || room < 256) {
      const int d = 4 * lane - c;              // the lane's first column is at d; past 3 there is none
      const bool one = d & 1, two = d & 2;
      const uint32_t lane_ok = d > 3 ? 0u : ~0u;
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const uint32_t keep = lane_ok & (ok >> i & 1u ? ~0u : 0u);
        if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int j = 0; j < 4; ++j) raw[i][j] = one ? (j < 3 ? raw[i][j + 1] : 0u) : raw[i][j];
#pragma unroll
          for (int j = 0; j < 4; ++j) raw[i][j] = two ? (j < 2 ? raw[i][j + 2] : 0u) : raw[i][j];
        } else {
          const uint64_t w = ((uint64_t)raw[i][1] << 32 | raw[i][0]) >> (16 * (d & 3));
          raw[i] = Raw{(uint32_t)w, (uint32_t)(w >> 32)};
        }
        raw[i] &= keep;
      }
    }
  }
  // bfloat16 stays packed: two values a word, their maxima and conversions too
  auto top = [&](int i, int w) { return raw[i][w] & (sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu); };
  if constexpr (ROWS) {
    uint8_t *data = p.data + b * p.rows * (p.kp / 2), *scale = p.scale + b * p.rows * (p.kp / 32);
    uint32_t keep[4];          // the byte of row 8 i + lane % 8 of the lane's block
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      uint32_t e[2];           // the largest exponents of the lane's blocks of rows i, i + 1
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
          e[k] = mx_max8<uint32_t>(max(max(top(i + k, 0), top(i + k, 1)), max(top(i + k, 2), top(i + k, 3)))) >> 23;
      } else {
        const uint32_t m0 = mx_max(top(i, 0), top(i, 1)), m1 = mx_max(top(i + 1, 0), top(i + 1, 1));
        const uint32_t m = mx_max8<v2h>(mx_max(mx_low(m0, m1), mx_high(m0, m1)));
        e[0] = m >> 7 & 255u;
        e[1] = m >> 23;
      }
      uint32_t q = 0u;         // row i's four values, then row i + 1's
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t byte = mx_byte(e[k]);
        const float s = mx_scale(byte);
        if constexpr (sizeof(T) == 4) {
          if (k == 0) { q = mx_cvt<0>(q, raw[i][0], raw[i][1], s); q = mx_cvt<1>(q, raw[i][2], raw[i][3], s); }
          else { q = mx_cvt<2>(q, raw[i + 1][0], raw[i + 1][1], s); q = mx_cvt<3>(q, raw[i + 1][2], raw[i + 1][3], s); }
        } else {
          if (k == 0) { q = mx_cvt<0>(q, raw[i][0], s); q = mx_cvt<1>(q, raw[i][1], s); }
          else { q = mx_cvt<2>(q, raw[i + 1][0], s); q = mx_cvt<3>(q, raw[i + 1][1], s); }
        }
        if (((i + k) & 7) == (lane & 7)) keep[i >> 3] = byte;
      }
      // even lanes write row i, odd ones row i + 1: their own values and the other's
      const uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)q, 0xB1, 0xF, 0xF, true);
      const uint32_t out = lane & 1 ? (other >> 16) | (q & 0xffff0000u) : (q & 0xffffu) | (other << 16);
      const int64_t r = r0 + i + (lane & 1);
      if (r < p.rows) *reinterpret_cast<uint32_t *>(data + r * (p.kp / 2) + cw / 2 + 4 * (lane >> 1)) = out;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t r = r0 + 8 * i + (lane & 7);
      if (r < p.rows) scale[r * (p.kp / 32) + c0 / 32] = (uint8_t)keep[i];
    }
  }
  if constexpr (ROWS && sizeof(T) == 2) {      // nothing of the above is kept in registers for the below
#pragma unroll
    for (int i = 0; i < 32; ++i) asm volatile("" : "+v"(raw[i]));
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t a = 0u, e;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 32; ++i) a = max(a, top(i, j));
      e = a >> 23;
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i) a = mx_max(a, top(i, j / 2));
      e = j & 1 ? a >> 23 : a >> 7 & 255u;
    }
    const uint32_t byte = mx_byte(e);
    const float s = mx_scale(byte);
    auto two = [&](auto sel, uint32_t q, int i) {        // rows i and i + 1 of the column
      if constexpr (sizeof(T) == 4) return mx_cvt<decltype(sel)::value>(q, raw[i][j], raw[i + 1][j], s);
      else return mx_cvt<decltype(sel)::value>(q, j & 1 ? mx_high(raw[i][j / 2], raw[i + 1][j / 2])
                                                        : mx_low(raw[i][j / 2], raw[i + 1][j / 2]), s);
    };
    v4u w;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t q = two(std::integral_constant<int, 0>{}, 0u, 8 * k);
      q = two(std::integral_constant<int, 1>{}, q, 8 * k + 2);
      q = two(std::integral_constant<int, 2>{}, q, 8 * k + 4);
      w[k] = two(std::integral_constant<int, 3>{}, q, 8 * k + 6);
    }
    const int c = 4 * lane + j;
    *reinterpret_cast<v4u *>(lds + c * 64 + 16 * (wave ^ (lane & 3))) = w;
    lds[256 * 64 + 4 * c + wave] = (uint8_t)byte;
  }
  __syncthreads();
  uint8_t *data = p.data_t + b * p.cols * (p.rp / 2), *scale = p.scale_t + b * p.cols * (p.rp / 32);
  const int64_t rw = r0 - 32 * wave;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int c = 64 * u + (threadIdx.x >> 2), k = threadIdx.x & 3;
    if (cw + c < p.cols)
      *reinterpret_cast<v4u *>(data + (cw + c) * (p.rp / 2) + rw / 2 + 16 * k) =
          *reinterpret_cast<const v4u *>(lds + c * 64 + 16 * (k ^ ((c >> 2) & 3)));
  }
  if (cw + threadIdx.x < p.cols)
    *reinterpret_cast<uint32_t *>(scale + (cw + threadIdx.x) * (p.rp / 32) + rw / 32) =
        *reinterpret_cast<const uint32_t *>(lds + 256 * 64 + 4 * threadIdx.x);
}

// Rows of a packed matrix, by an index: a wave per row, 16 bytes a lane (the scales 8).
__global__ __launch_bounds__(256) void mx4_gather(Mx4Mat x, int64_t x_rows, const int *__restrict__ row_index,
                                                  int64_t rows, int64_t kp, uint8_t *__restrict__ data,
                                                  uint8_t *__restrict__ scale) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int64_t r = (int64_t)blockIdx.x * 4 + wave; r < rows; r += (int64_t)gridDim.x * 4) {
    const int64_t src = row_index[r];
    const bool in = src >= 0 && src < x_rows;
    const v4u *from = reinterpret_cast<const v4u *>(x.data + (in ? src : 0) * (kp / 2));
    v4u *to = reinterpret_cast<v4u *>(data + r * (kp / 2));
    for (int64_t i = lane; i < kp / 32; i += 64) to[i] = in ? from[i] : v4u(0u);
    const v2u *sfrom = reinterpret_cast<const v2u *>(x.scale + (in ? src : 0) * (kp / 32));
    v2u *sto = reinterpret_cast<v2u *>(scale + r * (kp / 32));
    for (int64_t i = lane; i < kp / 256; i += 64) sto[i] = in ? sfrom[i] : v2u(0u);
  }
}

// The values of a packed matrix, along its rows as mx4_quantize_cols walks them: 16 bytes
// of values per lane, so that a wave's stores are contiguous (32 bytes of fp32 in two
// stores, each with gaps: 49 152 x 2048 177 us instead of 73), QC_UNITS independent loads
// at a time; the values, two to eight times the bytes read, are written past the L2s.
// Lanes of a row: 200 000 x 512 bfloat16 48 us with 16, 57 with 32, 75 with 64; 131 072 x
// 768 51 with 32, 73 with 64; 9000 x 11008 57 with 32, 47 with 64; fp32, half the values a
// lane, 200 000 x 512 67 with 32, 70 with 64, 131 072 x 768 75 with 32, 63 with 64.
template <typename T, int LPR>
__global__ __launch_bounds__(256) void mx4_dequantize(Mx4Mat a, int64_t rows, int64_t cols, int64_t kp,
                                                      T *__restrict__ out, int64_t ldo) {
  constexpr int ROWS = 256 / LPR, N = 16 / (int)sizeof(T);
  typedef typename std::conditional<N == 8, uint32_t, uint16_t>::type Codes;
  const int lane = threadIdx.x % LPR;
  for (int64_t r = (int64_t)blockIdx.x * ROWS + threadIdx.x / LPR; r < rows; r += (int64_t)gridDim.x * ROWS) {
    const uint8_t *dr = a.data + r * (kp / 2), *sr = a.scale + r * (kp / 32);
    T *o = out + r * ldo;
    for (int64_t c0 = N * lane; c0 < cols; c0 += QC_UNITS * LPR * N) {
      uint32_t q[QC_UNITS], byte[QC_UNITS];
#pragma unroll
      for (int u = 0; u < QC_UNITS; ++u) {
        const int64_t c = c0 + u * LPR * N;
        q[u] = byte[u] = 0u;
        if (c >= cols) continue;
        q[u] = *reinterpret_cast<const Codes *>(dr + c / 2);
        byte[u] = sr[c / 32];
      }
#pragma unroll
      for (int u = 0; u < QC_UNITS; ++u) {
        const int64_t c = c0 + u * LPR * N;
        if (c >= cols) continue;
        const float s = byte[u] == 255u ? __uint_as_float(0x7fc00000u) : mx_scale(byte[u]);
        float v[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
          // code m = 0, 1: 0.5 m; else (1 + 0.5 (m % 2)) 2^(m / 2 - 1)
          const uint32_t m = (q[u] >> (4 * j)) & 7u;
          const float f = m < 2u ? 0.5f * (float)m : __uint_as_float(((126u + (m >> 1)) << 23) | ((m & 1u) << 22));
          v[j] = ((q[u] >> (4 * j)) & 8u ? -f : f) * s;
        }
        if (c + N <= cols) {
          v4u w;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (N == 4) w[j] = __float_as_uint(v[j]);
            else w[j] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * j]) |
                        ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * j + 1]) << 16);
          }
          __builtin_nontemporal_store(w, reinterpret_cast<v4u_any *>(o + c));
        } else {
#pragma unroll
          for (int j = 0; j < N; ++j)
            if (c + j < cols) {
              if constexpr (N == 4) o[c + j] = v[j];
              else o[c + j] = __builtin_bit_cast(uint16_t, (__bf16)v[j]);
            }
        }
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
constexpr int MX_DEAL = 4;    // tiles of rows that grouped products deal to an XCD at a time

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

// Rows [0, rows) of a packed matrix (or of its scales), `bytes` each, as a buffer:
// loads past them give zeros.
constexpr int MX_RSRC_WORD3 = 0x00020000;    // raw 32-bit data
__device__ __forceinline__ __amdgpu_buffer_rsrc_t mx_buffer(const uint8_t *base, int rows, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(base), (short)0, (int)(uint32_t)(rows * bytes),
                                           MX_RSRC_WORD3);
}

// This workgroup's tile of a product by TM x TN: column tn, row tile in o.  Tiles
// that run together share operands in their XCD's L2: one product gives every XCD a
// contiguous run of tiles, eight tiles of rows by all tiles of columns at a time;
// groups, whose sizes differ (and whose last tiles may be none), are dealt to the
// XCDs in turn, four tiles of rows by all of columns.
template <int MODE, int TM>
__device__ __forceinline__ bool mx_my_tile(const MxParams &p, int &tn, int &g, MxTile &o) {
  const int x = blockIdx.x & 7, i = blockIdx.x >> 3;
  g = 0;
  int tm;
  if constexpr (MODE == MX_ONE) {
    const int nt = gridDim.x, per = nt >> 3, more = nt & 7, t = x * per + min(x, more) + i;
    const int per_group = 8 * p.tiles_n, group = t / per_group, first = group * 8;
    const int gsz = min(p.tiles_m - first, 8), in_group = t - group * per_group;
    tn = in_group / gsz;
    tm = first + in_group % gsz;
  } else {
    const int per = MX_DEAL * p.tiles_n, in = i % per, c = (i / per) * 8 + x;
    const int deals = (p.tiles_m + MX_DEAL - 1) / MX_DEAL;
    g = c / deals;
    tm = (c - g * deals) * MX_DEAL + in % MX_DEAL;
    tn = in / MX_DEAL;
    if (g >= (MODE == MX_K ? p.groups : 1) || tm >= p.tiles_m) return false;
  }
  return mx_tile<MODE, TM>(p, tm, g, o);
}

// The waves' results to C: register r of block (i, j) of a wave whose part of C
// starts at (row0, col0) is C[row0 + 32 i + xl][col0 + 32 j + 8 (r / 4) + 4 h + r % 4].
// `stage`: 32 rows of BJ * 32 values (16 bytes apart) of the wave's own.  STREAM: C is
// kept out of the L2s.
template <bool STREAM, typename T, int BI, int BJ>
__device__ __forceinline__ void mx_store(const MxParams &p, T *C, int64_t row0, int64_t row1, int64_t col0,
                                         uint8_t *stage, const v16f (&acc)[BI][BJ]) {
  constexpr int E = sizeof(T), STRIDE = BJ * 32 * E + 16, PER = 16 / E;
  const int lane = threadIdx.x & 63, xl = lane & 31, h = lane >> 5;
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
    constexpr int LANES = BJ * 32 / PER, RPI = 64 / LANES;       // lanes of a row, rows of an access
    const int er = lane / LANES, ec = PER * (lane % LANES);
#pragma unroll
    for (int u = 0; u < 32 / RPI; ++u) {
      const int x = er + RPI * u;
      const int64_t row = row0 + 32 * i + x, col = col0 + ec;
      const v4u v = *reinterpret_cast<const v4u *>(stage + x * STRIDE + ec * E);
      if (row >= row1 || col >= p.N) continue;
      T *dst = C + row * p.ldc + col;
      if (p.wide && col + PER <= p.N) {
        if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<v4u *>(dst));
        else *reinterpret_cast<v4u *>(dst) = v;
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

// One product by tiles of TM x TN through LDS: four waves (2 x 2), each
// (TM / 2) x (TN / 2) in blocks of 32 x 32.  K advances in slabs of 256 values (128
// bytes of a row, eight blocks, four matrix instructions of 64 values: lane (row,
// h) takes block 2 q + h at step q), two in LDS and a third on its way through
// registers.  Unit g (16 bytes) of row x lies at position g ^ (x / 2 % 8) of its 128
// bytes, so that sixteen consecutive rows of one unit are in different banks.  The
// scales come 16 bytes a row, two slabs' worth; byte q of the row's even or odd
// scales is step q's.
//
// One barrier a slab, before the last step, whose fragments are read by then: it
// makes the next slab visible and this one free.  From there to the next barrier
// every thread writes the units it holds of the slab after the next there and
// loads those of the one after that: each load has a whole slab's time, and reads,
// writes, loads and matrix instructions alternate evenly in the order written (one
// wave per SIMD: nothing else fills a gap, and a burst of loads holds the wave up
// until the L1 takes them, 27 cycles a kilobyte).  Loads into LDS without
// registers, which have to wait for the slab they replace: 4096 x 4096 x 14336
// 133 us; slabs of 128 values, four of them in LDS: 134 us (64 bytes of a row
// at a time take the L1 44 cycles a kilobyte).
//
// Slabs are whole in the packed rows; their padding's blocks get scales of 2^-127 on
// both sides, whose products vanish (and no NaN); loads past the last slab bring it
// again.
// Measured: 8192 x 14336 x 4096 252 us (3800 TFLOP/s), 4096 x 4096 x 14336 110 (4400), of one
// input again and again in a captured graph; over changing inputs in a kernel trace the first
// takes 258 to 290.  A loop of these instructions alone reaches 5600 on random data.  They are
// busy 0.50 of the time and waves wait 0.22 of it, at 1.75 to 1.9 GHz.
//
// The B operand goes first, so that a lane holds four consecutive columns of one
// row of C: results are rounded in registers, staged 32 rows at a time in the
// wave's part of the LDS and written 16 bytes a lane.
__device__ __forceinline__ void mx_sync() {      // this wave's LDS accesses done, then all waves'
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

template <int TM, int TN>
struct MxLds {
  static constexpr int ROWS = TM + TN;             // A's rows, then B's
  static constexpr int DATA = ROWS * 128, SCALE = ROWS * 16;
  static constexpr int BYTES = 2 * (DATA + SCALE);
};

template <typename T, int TM, int TN>
__global__ __launch_bounds__(256, TM == 256 ? 1 : 2) void mx4_gemm_tile(MxParams p) {
  typedef MxLds<TM, TN> L;
  constexpr int BI = TM / 64, BJ = TN / 64, NU = BI + BJ;
  constexpr int UNITS = L::ROWS / 32;              // units of a slab that a thread brings
  constexpr int SU = L::ROWS / 256;                // and rows of scales
  static_assert(UNITS == 2 * NU && BI * BJ % NU == 0, "a step's accesses pair up");
  __shared__ __attribute__((aligned(1024))) uint8_t lds[L::BYTES];
  int tn, g;
  MxTile o;
  mx_my_tile<MX_ONE, TM>(p, tn, g, o);
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

  const int am = (int)min((int64_t)TM, o.m1 - m0), bm = (int)min((int64_t)TN, p.N - n0);   // rows there are
  const int64_t srow = p.bytes / 16;
  const auto abuf = mx_buffer(p.A + m0 * p.bytes, am, p.bytes);
  const auto bbuf = mx_buffer(p.B + n0 * p.bytes, bm, p.bytes);
  const auto asbuf = mx_buffer(p.As + m0 * srow, am, srow);
  const auto bsbuf = mx_buffer(p.Bs + n0 * srow, bm, srow);
  // thread -> rows lr + 32 i, unit lg of A's and B's rows
  const int lr = tid >> 3, lg = tid & 7;
  const uint32_t off = (uint32_t)(lr * p.bytes + 16 * lg), row32 = (uint32_t)(32 * p.bytes);
  // and rows of scales tid + 256 i of A's and B's rows together
  uint32_t soff[SU];
#pragma unroll
  for (int i = 0; i < SU; ++i) {
    const int r = 256 * i + tid;
    soff[i] = (uint32_t)((r < TM ? r : r - TM) * srow);
  }
  const int slabs = (int)(p.bytes >> 7);           // of a packed row; at least 2
  const int s1 = (p.kb + 7) >> 3;                  // slabs that hold values
  const int dst = lr * 128 + 16 * (lg ^ ((lr >> 1) & 7));
  v4u r[UNITS], rs[SU];
  auto load = [&](int s, int i) {
    const int k = 128 * min(s, s1 - 1);
    if (i < TM / 32) r[i] = __builtin_amdgcn_raw_buffer_load_b128(abuf, (int)(off + i * row32), k, 0);
    else r[i] = __builtin_amdgcn_raw_buffer_load_b128(bbuf, (int)(off + (i - TM / 32) * row32), k, 0);
  };
  auto store = [&](int half, int i) {
    *reinterpret_cast<v4u *>(lds + half * L::DATA + i * 4096 + dst) = r[i];
  };
  // scales of the pair of slabs s and s + 1 (the last 16 bytes of a row if s is its last)
  auto load_scales = [&](int s) {
    const int at = 8 * min(s, slabs - 2);
#pragma unroll
    for (int i = 0; i < SU; ++i) {
      if (256 * i + 64 * wave < TM) rs[i] = __builtin_amdgcn_raw_buffer_load_b128(asbuf, (int)soff[i], at, 0);
      else rs[i] = __builtin_amdgcn_raw_buffer_load_b128(bsbuf, (int)soff[i], at, 0);
    }
  };
  auto store_scales = [&](int s) {
#pragma unroll
    for (int i = 0; i < SU; ++i)
      *reinterpret_cast<v4u *>(lds + 2 * L::DATA + ((s >> 1) & 1) * L::SCALE + (256 * i + tid) * 16) = rs[i];
  };

  v4u fa[2][BI], fb[2][BJ];
  uint32_t sa[2][BI], sb[2][BJ];                   // of a pair's first and second slab
  const int sw = (xl >> 1) & 7;
  const int arow = wm * (TM / 2) + xl, brow = TM + wn * (TN / 2) + xl;
  const uint32_t pick = h ? 0x07050301u : 0x06040200u;
  // fragment x of a step, in the order the matrix instructions want them
  auto frag = [&](int f, int half, int q, int x) {
    const uint8_t *d = lds + half * L::DATA + 16 * ((2 * q + h) ^ sw);
    if (x == 0 || x > BJ) {
      const int i = x ? x - BJ : 0;
      fa[f][i] = *reinterpret_cast<const v4u *>(d + (arow + 32 * i) * 128);
    } else {
      fb[f][x - 1] = *reinterpret_cast<const v4u *>(d + (brow + 32 * (x - 1)) * 128);
    }
  };
  auto scales = [&](int f, int s) {
    const int pair = s & ~1;
    const uint8_t *d = lds + 2 * L::DATA + ((s >> 1) & 1) * L::SCALE + 8 * min(s - min(pair, slabs - 2), 1);
    uint32_t mine = 0u;                            // bytes of the blocks that hold values
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int kb = 8 * s + 2 * q + h;
      mine |= kb < p.kb ? 0xffu << (8 * q) : 0u;
    }
#pragma unroll
    for (int i = 0; i < BI; ++i) {
      const uint2 v = *reinterpret_cast<const uint2 *>(d + (arow + 32 * i) * 16);
      sa[f][i] = __builtin_amdgcn_perm(v.y, v.x, pick) & mine;
    }
#pragma unroll
    for (int j = 0; j < BJ; ++j) {
      const uint2 v = *reinterpret_cast<const uint2 *>(d + (brow + 32 * j) * 16);
      sb[f][j] = __builtin_amdgcn_perm(v.y, v.x, pick) & mine;
    }
  };
  using std::integral_constant;
  // Step Q of a pair's slab P: multiplies fragment set Q % 2, reads the other, of the
  // next step, and moves a quarter of the units on: of slab ws to LDS, of slab ws + 1
  // from memory.
  auto step = [&](auto qc, auto par, int ws) {
    constexpr int Q = decltype(qc)::value, P = decltype(par)::value, f = Q & 1;
    constexpr int rh = Q == 3 ? P ^ 1 : P, rq = (Q + 1) & 3, wh = rh ^ 1, first = rq * NU / 2;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      frag(f ^ 1, rh, rq, u);
      if ((u & 1) == 0) {
        store(wh, first + u / 2);
        load(ws + 1, first + u / 2);
      }
#pragma unroll
      for (int v = 0; v < BI * BJ / NU; ++v) {
        const int k = u * (BI * BJ / NU) + v, i = k / BJ, j = k % BJ;
        const v4u a = fa[f][i], b = fb[f][j];
        const v8i va = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
        const v8i vb = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(vb, va, acc[i][j], 4, 4, Q, (int)sb[P][j], Q,
                                                                    (int)sa[P][i]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto slab = [&](auto par, int s) {
    constexpr int P = decltype(par)::value;
    step(integral_constant<int, 0>{}, par, s + 1);
    step(integral_constant<int, 1>{}, par, s + 1);
    step(integral_constant<int, 2>{}, par, s + 1);
    mx_sync();
    scales(P ^ 1, s + 1);
    if constexpr (P == 0) {
      store_scales(s + 2);
      load_scales(s + 4);
    }
    step(integral_constant<int, 3>{}, par, s + 2);
  };
  if (s1 > 0) {
    load_scales(0);
#pragma unroll
    for (int i = 0; i < UNITS; ++i) load(0, i);
    store_scales(0);
    load_scales(2);
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      store(0, i);
      load(1, i);
    }
    mx_sync();
    scales(0, 0);
#pragma unroll
    for (int u = 0; u < NU; ++u) frag(0, 0, 0, u);
#pragma unroll
    for (int i = 0; i < NU / 2; ++i) {
      store(1, i);
      load(2, i);
    }
    for (int s = 0; s < s1; s += 2) {
      slab(integral_constant<int, 0>{}, s);
      slab(integral_constant<int, 1>{}, s + 1);
    }
  }

  constexpr int STRIDE = BJ * 32 * (int)sizeof(T) + 16;
  static_assert(4 * 32 * STRIDE <= L::BYTES, "the staged rows fit the LDS");
  mx_sync();
  mx_store<TM == 256, T, BI, BJ>(p, static_cast<T *>(p.C), m0 + wm * (TM / 2), o.m1, n0 + wn * (TN / 2),
                      lds + wave * 32 * STRIDE, acc);
}

// Tiles of 128 x 128 for products of fewer or shorter tiles: one slab in LDS, the
// next on its way through registers, and four workgroups per compute unit, which cover
// each other's barriers, first loads and epilogues.  Groups by rows (64 experts of 2048
// x 768, 512 rows each) 45 to 58 us in a kernel trace, matrix instructions busy 0.35 of it and
// waves waiting 0.36 of theirs; by k (their gradients) 94 to 105 us, busy 0.21: bound by the
// 403 MB written.  Nothing splits a group's sum over workgroups: 2 groups of 64 x 64, 2048 k
// each, take 10 us on two compute units, 512 x 512 x 65536 79 us on 16 (in the tiles above).
template <int MODE, typename T, bool STREAM>
__global__ __launch_bounds__(256, 4) void mx4_gemm_tile128(MxParams p) {
  constexpr int TM = 128, TN = 128, BI = 2, BJ = 2, UNITS = 8, DATA = 256 * 128;
  __shared__ __attribute__((aligned(16))) uint8_t lds[DATA + 256 * 8];
  int tn, g;
  MxTile o;
  if (!mx_my_tile<MODE, TM>(p, tn, g, o)) return;
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
  const int am = (int)min((int64_t)TM, o.m1 - m0), bm = (int)min((int64_t)TN, p.N - n0);   // rows there are
  const int64_t srow = p.bytes / 16;
  const auto abuf = mx_buffer(p.A + m0 * p.bytes, am, p.bytes);
  const auto bbuf = mx_buffer(p.B + (o.b0 + n0) * p.bytes, bm, p.bytes);
  // thread -> rows lr + 32 i, unit lg of A's and B's rows; its row of scales
  const int lr = tid >> 3, lg = tid & 7;
  const uint32_t off = (uint32_t)(lr * p.bytes + 16 * lg), row32 = (uint32_t)(32 * p.bytes);
  const bool of_a = wave < TM / 64;
  const auto sbuf = of_a ? mx_buffer(p.As + m0 * srow, am, srow) : mx_buffer(p.Bs + (o.b0 + n0) * srow, bm, srow);
  const uint32_t soff = (uint32_t)((of_a ? tid : tid - TM) * srow);
  const int s0 = o.kb0 >> 3, s1 = o.kb1 > o.kb0 ? (o.kb1 + 7) >> 3 : s0;
  const int dst = lr * 128 + 16 * (lg ^ ((lr >> 1) & 7));
  v4u r[UNITS];
  v2u rs;
  auto load = [&](int s) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_raw_buffer_load_b128(abuf, (int)(off + i * row32), 128 * s, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      r[4 + i] = __builtin_amdgcn_raw_buffer_load_b128(bbuf, (int)(off + i * row32), 128 * s, 0);
    rs = __builtin_amdgcn_raw_buffer_load_b64(sbuf, (int)soff, 8 * s, 0);
  };
  if (s1 > s0) load(s0);
  const int sw = (xl >> 1) & 7, arow = wm * 64 + xl, brow = TM + wn * 64 + xl;
  const uint32_t pick = h ? 0x07050301u : 0x06040200u;
  for (int s = s0; s < s1; ++s) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < UNITS; ++i) *reinterpret_cast<v4u *>(lds + i * 4096 + dst) = r[i];
    *reinterpret_cast<v2u *>(lds + DATA + 8 * tid) = rs;
    __syncthreads();
    load(min(s + 1, s1 - 1));
    uint32_t mine = 0u;                            // bytes of the blocks that are this product's
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int kb = 8 * s + 2 * q + h;
      mine |= kb >= o.kb0 && kb < o.kb1 ? 0xffu << (8 * q) : 0u;
    }
    uint32_t sa[BI], sb[BJ];
#pragma unroll
    for (int i = 0; i < BI; ++i) {
      const uint2 v = *reinterpret_cast<const uint2 *>(lds + DATA + 8 * (arow + 32 * i));
      sa[i] = __builtin_amdgcn_perm(v.y, v.x, pick) & mine;
    }
#pragma unroll
    for (int j = 0; j < BJ; ++j) {
      const uint2 v = *reinterpret_cast<const uint2 *>(lds + DATA + 8 * (brow + 32 * j));
      sb[j] = __builtin_amdgcn_perm(v.y, v.x, pick) & mine;
    }
    auto step = [&](auto qc) {
      constexpr int q = decltype(qc)::value;
      const uint8_t *d = lds + 16 * ((2 * q + h) ^ sw);
      v4u a[BI], b[BJ];
#pragma unroll
      for (int i = 0; i < BI; ++i) a[i] = *reinterpret_cast<const v4u *>(d + (arow + 32 * i) * 128);
#pragma unroll
      for (int j = 0; j < BJ; ++j) b[j] = *reinterpret_cast<const v4u *>(d + (brow + 32 * j) * 128);
#pragma unroll
      for (int i = 0; i < BI; ++i)
#pragma unroll
        for (int j = 0; j < BJ; ++j) {
          const v8i va = {(int)a[i].x, (int)a[i].y, (int)a[i].z, (int)a[i].w, 0, 0, 0, 0};
          const v8i vb = {(int)b[j].x, (int)b[j].y, (int)b[j].z, (int)b[j].w, 0, 0, 0, 0};
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(vb, va, acc[i][j], 4, 4, q, (int)sb[j], q,
                                                                      (int)sa[i]);
        }
    };
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 3>{});
  }
  constexpr int STRIDE = BJ * 32 * (int)sizeof(T) + 16;
  static_assert(4 * 32 * STRIDE <= (int)sizeof(lds), "the staged rows fit the LDS");
  __syncthreads();
  mx_store<STREAM, T, BI, BJ>(p, static_cast<T *>(p.C) + o.c0, m0 + wm * 64, o.m1, n0 + wn * 64,
                      lds + wave * 32 * STRIDE, acc);
}

// Few rows: 32 x 32 of C per workgroup, whose MXF_W waves take the slabs of K in turn
// and add their sums in LDS in order.  Operands go from memory to registers, all of a
// wave's loads of MXF_AHEAD slabs ahead of its matrix instructions; B is read once, by
// as many waves as there are: 16 x 14336 x 4096 11.6 us in a kernel trace over changing
// weights, 2.7 TB/s of them, 10.2 where the last-level cache has them, first loads and the
// join of the waves' sums included (a launch alone takes 3).
constexpr int MXF_W = 8, MXF_AHEAD = 2;
template <int MODE, typename T>
__global__ __launch_bounds__(64 * MXF_W) void mx4_gemm_few(MxParams p) {
  __shared__ float part[MXF_W][16][64];
  MxTile o;
  const int64_t tm = blockIdx.x / p.tiles_n, tn = blockIdx.x - tm * p.tiles_n;
  if (!mx_tile<MODE, 32>(p, tm, 0, o)) return;
  const int64_t m0 = o.m0, n0 = tn * 32;
  if (m0 >= o.m1) return;
  const int tid = threadIdx.x, lane = tid & 63, xl = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int am = (int)min((int64_t)32, o.m1 - m0), bm = (int)min((int64_t)32, p.N - n0);   // rows there are
  const int64_t srow = p.bytes / 16;
  const auto abuf = mx_buffer(p.A + m0 * p.bytes, am, p.bytes);
  const auto bbuf = mx_buffer(p.B + (o.b0 + n0) * p.bytes, bm, p.bytes);
  const auto asbuf = mx_buffer(p.As + m0 * srow, am, srow);
  const auto bsbuf = mx_buffer(p.Bs + (o.b0 + n0) * srow, bm, srow);
  const int off = (int)(uint32_t)(xl * p.bytes + 16 * h), soff = (int)(uint32_t)(xl * srow);
  const uint32_t pick = h ? 0x07050301u : 0x06040200u;
  const int s1 = o.kb1 > o.kb0 ? (o.kb1 + 7) >> 3 : 0;     // kb0 is 0 where K is not grouped
  v16f acc;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0.f;
  for (int s0 = wave; s0 < s1; s0 += MXF_W * MXF_AHEAD) {
    v4u a[MXF_AHEAD][4], b[MXF_AHEAD][4];
    v2u za[MXF_AHEAD], zb[MXF_AHEAD];
#pragma unroll
    for (int d = 0; d < MXF_AHEAD; ++d) {
      const int s = min(s0 + d * MXF_W, s1 - 1);
#pragma unroll
      for (int q = 0; q < 4; ++q) b[d][q] = __builtin_amdgcn_raw_buffer_load_b128(bbuf, off + 32 * q, 128 * s, 0);
#pragma unroll
      for (int q = 0; q < 4; ++q) a[d][q] = __builtin_amdgcn_raw_buffer_load_b128(abuf, off + 32 * q, 128 * s, 0);
      za[d] = __builtin_amdgcn_raw_buffer_load_b64(asbuf, soff, 8 * s, 0);
      zb[d] = __builtin_amdgcn_raw_buffer_load_b64(bsbuf, soff, 8 * s, 0);
    }
#pragma unroll
    for (int d = 0; d < MXF_AHEAD; ++d) {
      const int s = s0 + d * MXF_W;
      uint32_t mine = 0u;                          // bytes of the blocks that hold values
#pragma unroll
      for (int q = 0; q < 4; ++q) mine |= 8 * s + 2 * q + h < o.kb1 ? 0xffu << (8 * q) : 0u;
      const uint32_t sa = __builtin_amdgcn_perm(za[d].y, za[d].x, pick) & mine;
      const uint32_t sb = __builtin_amdgcn_perm(zb[d].y, zb[d].x, pick) & mine;
      auto step = [&](auto qc) {
        constexpr int q = decltype(qc)::value;
        const v8i va = {(int)a[d][q].x, (int)a[d][q].y, (int)a[d][q].z, (int)a[d][q].w, 0, 0, 0, 0};
        const v8i vb = {(int)b[d][q].x, (int)b[d][q].y, (int)b[d][q].z, (int)b[d][q].w, 0, 0, 0, 0};
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(va, vb, acc, 4, 4, q, (int)sa, q, (int)sb);
      };
      step(std::integral_constant<int, 0>{});
      step(std::integral_constant<int, 1>{});
      step(std::integral_constant<int, 2>{});
      step(std::integral_constant<int, 3>{});
    }
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) part[wave][r][lane] = acc[r];
  __syncthreads();
  // register r of lane (xl, h) is C[8 (r / 4) + 4 h + r % 4][xl]
  T *C = static_cast<T *>(p.C);
#pragma unroll
  for (int e = tid; e < 1024; e += 64 * MXF_W) {
    const int y = e >> 5, x = e & 31, r = 4 * (y >> 3) + (y & 3), l = x + 32 * ((y >> 2) & 1);
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < MXF_W; ++w) v += part[w][r][l];
    if (m0 + y >= o.m1 || n0 + x >= p.N) continue;
    T *c = C + (m0 + y) * p.ldc + n0 + x;
    if constexpr (sizeof(T) == 4) *c = v;
    else *c = __builtin_bit_cast(uint16_t, (__bf16)v);
  }
}

// Gradients larger than the L2s (32 MB) are written past them: through them, one of
// 403 MB pushed its operands out, 180 us against 105; one that fits is found there by
// its reader.  The outputs of 256-tiles are about as large or larger.
constexpr int64_t MX_L2 = 32 << 20;

// Few rows: 32 x 32 tiles, against 128-tiles, microseconds of the one / the other.
//
// While the tiles are no more than the compute units: 256 tiles of 16 rows, K = 512 3.2 /
// 4.5, 2048 5.6 / 7.2, 4096 6.6 / 10.9, 14336 19 / 30; of 128 rows 3.6 / 4.9, 6.6 / 7.6,
// 7.2 / 11, 20 / 30.  With 288 tiles of 32 rows and more it is over from K = 1024 on (6.3 /
// 5.6, K = 4096 12.1 / 11.2).
//
// For at most mx_few_rows rows, up to twice as many: the eight waves load 16 slabs of 256
// at a time, and where K fills those badly or has many of them only fewer rows pay.  400
// tiles, every step of K below for 2, 4 .. 16 rows: K to 1280 3.8 / 4.5 (512, 8 rows) to 6.4 / 6.5
// (1280, 16); 2048 7.5 / 7.2 at 2 rows, 8.9 / 7.4 at 16; 2560 7.8 / 8.2 at 8, 8.6 / 8.3 at 16; 2816
// to 4864 9.4 / 11.3 at 8, 10.5 / 11.2 at 16 (4096); 5120 to 15360 12.8 / 13.3 (5120), 24.8 / 22.7
// (10240) and 25.8 / 26.6 (12288) at 8, 14.5 / 13.6 to 36 / 30 at 16; 16384 35 / 34 at 2.
constexpr int64_t MX_FEW = 256;
int64_t mx_few_rows(int64_t slabs) {
  if (slabs <= 5 || (slabs >= 11 && slabs <= 19)) return 16;
  if (slabs == 8 || slabs > 60) return 0;
  return slabs < 8 ? 4 : 8;
}
// Grouped rows: the launch has a row of tiles more for every group, which may have none, and
// stays below MX_FEW_GROUPED tiles (64 experts of 2048 x 768, 8 of them a token: 4 tokens, 2328
// tiles, 16 / 10).  The groups' rows fill at most M / 32 rows of tiles.  For K past 2560 the small
// tiles win up to about 900 filled ones, whatever N (2 of 8 experts of 4096 x 1024: 768 18.5 / 23.1;
// 2 of 4: 1152 27 / 24); for less K up to 500 where N is 256, 750 to 1000 where it is 2048 (2 of 4
// to 16 experts of 2048 x 768: 384 11.1 / 10.7, 864 19.6 / 11.3; of 1024 x 512: 512 7.1 / 7.3, 768
// 9.2 / 7.5).  Over 2002 shapes (4 to 64 experts, 1 to 512 tokens, K 256 to 7168, N 256 to 4096)
// this takes 0.5 per cent longer than the better of the two, 31 at worst; by MX_FEW_GROUPED alone
// 2.7 and 99.
constexpr int64_t MX_FEW_GROUPED = 1536;
bool mx_few_grouped(int64_t launched, int64_t filled, int64_t tiles_n, int64_t slabs) {
  return launched <= MX_FEW_GROUPED && filled <= (slabs >= 11 ? 896 : std::min<int64_t>(768, 448 + 6 * tiles_n));
}
// 256 x 256 where they fill 0.8 of the rounds of one a compute unit that they take:
// 4096 x 4096 x 14336 (1.0) 117 us against 155 in 128-tiles, 6000 x 5000 x 4096 (0.9) 75
// against 85, 32768 x 768 x 2048 (0.75) 40 against 37, 16384 x 1100 x 4096 (0.5) 86
// against 77, 512 x 14336 x 4096 (0.4) 38 against 25.  Grouped products leave the last
// tile of a group part empty and have few slabs: 128-tiles, four workgroups a compute
// unit (the weight gradients of 64 experts of 2048 x 768, 512 rows each, 105 us; with
// two and two slabs in LDS 125 to 138).
constexpr int64_t MX_CUS = 256;

template <int MODE, typename T>
hipError_t mx_launch(MxParams p, hipStream_t s) {
  auto tiles = [&](int bt) -> int64_t {
    const int64_t tm = (p.M + bt - 1) / bt + (MODE == MX_ROWS ? p.groups + 1 : 0), tn = (p.N + bt - 1) / bt;
    p.tiles_m = (int)tm;
    p.tiles_n = (int)tn;
    if (MODE == MX_ONE || bt == 32) return tm * tn;
    const int64_t deals = (tm + MX_DEAL - 1) / MX_DEAL * (MODE == MX_K ? p.groups : 1);
    return (deals + 7) / 8 * 8 * MX_DEAL * tn;
  };
  int64_t n;
  if constexpr (MODE != MX_K) {
    n = tiles(32);
    const int64_t slabs = p.bytes / 128;
    if (MODE == MX_ROWS ? mx_few_grouped(n, (p.M + 31) / 32 * p.tiles_n, p.tiles_n, slabs)
                        : n <= (p.M <= mx_few_rows(slabs) ? 2 * MX_FEW : MX_FEW)) {
      hipLaunchKernelGGL((mx4_gemm_few<MODE, T>), dim3((unsigned)n), dim3(64 * MXF_W), 0, s, p);
      return hipGetLastError();
    }
  }
  if constexpr (MODE == MX_ONE) {
    if (p.bytes >= 256) {                  // a load of scales brings two slabs'
      n = tiles(256);
      const double rounds = (double)((n + MX_CUS - 1) / MX_CUS * MX_CUS) * 65536.0;
      if ((double)p.M * (double)p.N >= 0.8 * rounds) {
        hipLaunchKernelGGL((mx4_gemm_tile<T, 256, 256>), dim3((unsigned)n), dim3(256), 0, s, p);
      } else {
        n = tiles(128);
        hipLaunchKernelGGL((mx4_gemm_tile<T, 128, 128>), dim3((unsigned)n), dim3(256), 0, s, p);
      }
      return hipGetLastError();
    }
  }
  n = tiles(128);
  if (n > INT32_MAX) return hipErrorInvalidValue;
  if constexpr (MODE == MX_K) {
    if (p.groups * p.sC * (int64_t)sizeof(T) > MX_L2) {
      hipLaunchKernelGGL((mx4_gemm_tile128<MODE, T, true>), dim3((unsigned)n), dim3(256), 0, s, p);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((mx4_gemm_tile128<MODE, T, false>), dim3((unsigned)n), dim3(256), 0, s, p);
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
  if (!d.data_t) {
    if (d.rows == 0) return hipSuccess;
    const int lanes = mx_lanes(p.kp, 512, 1024), rows = 256 / lanes;
    const dim3 grid((unsigned)std::min<int64_t>((d.rows + rows - 1) / rows, 1 << 16), (unsigned)d.batch);
#define SOAP_MXQ(T, L) \
  if (lanes == L) hipLaunchKernelGGL((mx4_quantize_cols<T, L>), grid, dim3(256), 0, s, p)
    if (d.bf16) { SOAP_MXQ(uint16_t, 16); SOAP_MXQ(uint16_t, 32); SOAP_MXQ(uint16_t, 64); }
    else { SOAP_MXQ(float, 16); SOAP_MXQ(float, 32); SOAP_MXQ(float, 64); }
#undef SOAP_MXQ
    return hipGetLastError();
  }
  const int64_t tiles = (p.rp / 128) * (p.kp / 256);
  if (tiles == 0) return hipSuccess;
  if (tiles > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid((unsigned)tiles, (unsigned)d.batch);
#define SOAP_MXQ(T, R)                                                                                    \
  do {                                                                                                    \
    if (d.row_index) hipLaunchKernelGGL((mx4_quantize_tile<T, R, true>), grid, dim3(256), 0, s, p);       \
    else hipLaunchKernelGGL((mx4_quantize_tile<T, R, false>), grid, dim3(256), 0, s, p);                  \
  } while (0)
  if (d.bf16) { if (d.data) SOAP_MXQ(uint16_t, true); else SOAP_MXQ(uint16_t, false); }
  else { if (d.data) SOAP_MXQ(float, true); else SOAP_MXQ(float, false); }
#undef SOAP_MXQ
  return hipGetLastError();
}

hipError_t launch_mx4_gather(const Mx4Mat &x, int64_t x_rows, const int *row_index, int64_t rows,
                             int64_t k, uint8_t *data, uint8_t *scale, hipStream_t s) {
  if (rows <= 0) return hipSuccess;
  const dim3 grid((unsigned)std::min<int64_t>((rows + 3) / 4, 1 << 16));
  hipLaunchKernelGGL(mx4_gather, grid, dim3(256), 0, s, x, x_rows, row_index, rows, mx4_padded(k), data, scale);
  return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const Mx4Mat &a, int64_t rows, int64_t cols, bool bf16, void *out,
                                 int64_t ldo, hipStream_t s) {
  if (rows <= 0) return hipSuccess;
  const int64_t kp = mx4_padded(cols);
  const int lanes = bf16 ? mx_lanes(kp, 512, 2304) : mx_lanes(kp, 256, 512), per = 256 / lanes;
  const dim3 grid((unsigned)std::min<int64_t>((rows + per - 1) / per, 1 << 16));
#define SOAP_MXV(T, L)                                                                                  \
  if (lanes == L)                                                                                       \
  hipLaunchKernelGGL((mx4_dequantize<T, L>), grid, dim3(256), 0, s, a, rows, cols, kp, static_cast<T *>(out), ldo)
  if (bf16) { SOAP_MXV(uint16_t, 16); SOAP_MXV(uint16_t, 32); SOAP_MXV(uint16_t, 64); }
  else { SOAP_MXV(float, 16); SOAP_MXV(float, 32); SOAP_MXV(float, 64); }
#undef SOAP_MXV
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
