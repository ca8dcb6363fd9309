// The gated feed-forward block and its gradients in bfloat16, sums in fp32:
//
//   G = X Wg,  U = X Wu,  H = act(G) * U,  Y = H Wd
//   dH = dY Wd^T,  dG = dH * U * act'(G),  dU = dH * act(G)
//   dX = dG Wg^T + dU Wu^T,  dWg = X^T dG,  dWu = X^T dU,  dWd = H^T dY
//
// X is tokens x m, Wg and Wu m x n, Wd n x p.  H, dG and dU are rounded to bfloat16 once, as
// the operands of the next product; act works on fp32 sums forward and on the kept (rounded)
// G and U backward.
//
// Every product is one kernel, product_tiles: C = sum over k of A(x, k) B(y, k), its operands
// in memory either k-contiguous ([x][k]: X, H, dY, dG, dU, and the weights seen from their
// rows) or x-contiguous ([k][x]: the weights forward, and both operands of the weights'
// gradients), so that nothing is transposed beforehand.  Both come to LDS as they are in
// memory, by loads that write LDS themselves, in blocks of 64 rows of 128 bytes, 16-byte units
// permuted within a row so that no two of a read's lanes meet in a bank: k-contiguous
// blocks are read 16 bytes of a row at a time, x-contiguous ones by the transposing reads,
// which give a lane four k of its own x.
//
// Operands past their ends read as zeros (buffer bounds; units past the end of k are sent
// out of bounds), so that sizes need no multiple of a tile; m, n and p are multiples of 8
// and rows 16-byte aligned, so that no unit crosses an end.
#include "soap.h"

#include "internal.h"

#include <algorithm>

namespace soap {
namespace {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) v4s lds_v4s;
typedef __attribute__((address_space(3))) void lds_void;

constexpr int GP_THREADS = 256, GP_KB = 64;      // four waves; k of a slab
constexpr int GP_BLOCK = 64 * 128;               // bytes of a block of 64 rows in LDS
constexpr int GP_RSRC = 0x00020000;              // raw 32-bit data

enum { GP_BF16, GP_F32, GP_GATED, GP_DGATED, GP_PART };

struct GpParams {
  int M, N, K;                 // N: of one matrix; K: of one segment
  const uint16_t *A[2], *B[2]; // B[1]: up's weights or gradients; A[1]: the second segment of k
  int64_t lda, ldb;
  int segments;                // of k, each with operands of its own
  int tiles_m, tiles_n, pairs; // pairs: B and C by the tile's column (the second half: [1])
  void *C[2];
  int64_t ldc;
  // gated: C[0] the product, kept G and U (or null); dgated: C[0] = dG, C[1] = dU, H
  const uint16_t *gate, *up;
  uint16_t *keep_gate, *keep_up, *hidden;
  int act;
};

__device__ __forceinline__ uint16_t gp_round(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ float gp_float(uint16_t h) { return __uint_as_float((uint32_t)h << 16); }

// The activation and, for the gradient, its derivative.
__device__ __forceinline__ float gp_act(float x, int act) {
  if (act == SOAP_ACT_SILU) return x / (1.f + expf(-x));
  return 0.5f * x * (1.f + erff(x * 0.70710678118654752440f));
}
__device__ __forceinline__ float gp_dact(float x, int act) {
  if (act == SOAP_ACT_SILU) {
    const float s = 1.f / (1.f + expf(-x));
    return s * (1.f + x * (1.f - s));
  }
  return 0.5f * (1.f + erff(x * 0.70710678118654752440f)) + x * 0.39894228040143267794f * expf(-0.5f * x * x);
}

// What one operand's blocks of a slab are loaded from: rows of its matrix from the tile's
// first on, `left` bytes to the matrix' end.
struct GpSource {
  const char *base;
  int64_t left;
};
__device__ __forceinline__ void gp_load(const GpSource &s, uint8_t *lds, uint32_t offset) {
  const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(s.base), (short)0,
                                                   (int)(uint32_t)min(max(s.left, (int64_t)0), (int64_t)0xfffffff0), GP_RSRC);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void *)lds, 16, (int)offset, 0, 0, 0);
}

// NB: blocks of 32 x 32 on a side of a wave's share; tiles of 64 NB.
template <bool AK, bool BK, int EPI, int NB>
__global__ __launch_bounds__(GP_THREADS, NB == 4 ? 1 : 2) void product_tiles(GpParams p) {
  constexpr int TB = 64 * NB, SUB = TB / 64, OP = SUB * GP_BLOCK, LOADS = 2 * SUB;
  constexpr int SLD = TB + 4;                    // staging row of the epilogue, floats
  constexpr int BAND = 64;
  static_assert(BAND * SLD * 4 <= 4 * OP, "the epilogue's band fits the slabs");
  __shared__ __attribute__((aligned(1024))) uint8_t lds[4 * OP];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1, xl = lane & 31, h = lane >> 5;

  // the tile: a contiguous run for each XCD, eight tiles of rows by all columns at a time
  int tm, tn;
  {
    const int nt = p.tiles_m * p.tiles_n, q = nt >> 3, r = nt & 7, x = blockIdx.x & 7;
    const int t = x * q + min(x, r) + (blockIdx.x >> 3);
    const int group = t / (8 * p.tiles_n), first = 8 * group, size = min(p.tiles_m - first, 8);
    const int in = t - group * 8 * p.tiles_n;
    tm = first + in % size;
    tn = in / size;
  }
  int which = 0;
  if (p.pairs) {
    const int half = p.tiles_n >> 1;
    which = tn >= half;
    tn -= which ? half : 0;
  }
  constexpr bool TWO = EPI == GP_GATED;          // columns of both matrices, 64 by 64
  const int m0 = tm * TB, n0 = tn * (TWO ? TB / 2 : TB);
  const int64_t lda2 = 2 * p.lda, ldb2 = 2 * p.ldb;

  // a wave's loads: of block j >> 3 the rows 8 (j & 7) .., j = wave + 4 i
  uint32_t offa[LOADS], offb[LOADS];
  int ua[2], ub[2];                              // the k unit that a lane's loads begin at
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int j = wave + 4 * i, s = j >> 3, row = 8 * (j & 7) + (lane >> 3);
    const int uk = (lane & 7) ^ ((row >> 1) & 7), ux = (lane & 7) ^ (4 * ((row >> 1) & 1));
    offa[i] = AK ? (uint32_t)((64 * s + row) * lda2) + 16 * uk : (uint32_t)(row * lda2) + 128 * s + 16 * ux;
    const int sb = TWO ? s >> 1 : s;
    offb[i] = BK ? (uint32_t)((64 * sb + row) * ldb2) + 16 * uk : (uint32_t)(row * ldb2) + 128 * sb + 16 * ux;
  }
  ua[0] = ub[0] = (lane & 7) ^ ((8 * (wave & 7) + (lane >> 3)) >> 1 & 7);
  ua[1] = ub[1] = ua[0];                         // rows 32 apart permute alike
  const int nk1 = (p.K + GP_KB - 1) / GP_KB, nk = nk1 * p.segments;

  auto load = [&](int kt) {
    const int seg = kt >= nk1, k0 = (kt - seg * nk1) * GP_KB;
    uint8_t *la = lds + (kt & 1) * 2 * OP, *lb = la + OP;
    auto source = [&](const uint16_t *q, bool kc, int x0, int X, int64_t ld2) {
      GpSource s;
      if (kc) {
        s.base = (const char *)q + x0 * ld2 + 2 * k0;
        s.left = (X - x0 - 1) * ld2 + 2 * (p.K - k0);
      } else {
        s.base = (const char *)q + k0 * ld2 + 2 * x0;
        s.left = (p.K - k0 - 1) * ld2 + 2 * (X - x0);
      }
      return s;
    };
    const GpSource a = source(p.A[seg], AK, m0, p.M, lda2);
    const GpSource b0 = source(p.B[TWO ? 0 : p.segments > 1 ? seg : which], BK, n0, p.N, ldb2);
    const GpSource b1 = TWO ? source(p.B[1], BK, n0, p.N, ldb2) : b0;
    const bool dead = k0 + 8 * ua[0] >= p.K;     // a unit of k past the end
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int j = wave + 4 * i, s = j >> 3;
      gp_load(a, la + j * 1024, AK && dead ? 0xfffffff0u : offa[i]);
      gp_load(TWO && (s & 1) ? b1 : b0, lb + j * 1024, BK && dead ? 0xfffffff0u : offb[i]);
    }
  };

  // fragments: the 8 k from 16 q + 8 h on of row `x` (a multiple of 32, and the lane's)
  auto frag = [&](const uint8_t *op, bool kc, int x, int q) -> v8bf {
    const uint8_t *b = op + (x >> 6) * GP_BLOCK;
    if (kc) {
      const int r = (x & 32) + xl;
      return *reinterpret_cast<const v8bf *>(b + r * 128 + 16 * ((2 * q + h) ^ ((r >> 1) & 7)));
    }
    const int i = lane & 15, r = i >> 2, u = (x & 32) / 8 + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
    const uint8_t *at = b + (16 * q + 8 * h + r) * 128 + 16 * (u ^ (4 * (r >> 1))) + 8 * (i & 1);
    const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)at);
    const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(at + 4 * 128));
    return __builtin_bit_cast(v8bf, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };

  v16f acc[NB][NB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  if (nk) load(0);
  for (int kt = 0; kt < nk; ++kt) {
    __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0)
    __syncthreads();
    if (kt + 1 < nk) load(kt + 1);
    const uint8_t *la = lds + (kt & 1) * 2 * OP, *lb = la + OP;
#pragma unroll
    for (int q = 0; q < GP_KB / 16; ++q) {
      v8bf fa[NB], fb[NB];
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        fa[i] = frag(la, AK, wm * 32 * NB + 32 * i, q);
        // gated: the first half of a wave's columns are the gate's, in block 2 w, then up's in 2 w + 1
        fb[i] = TWO && NB == 2 ? frag(lb, BK, 64 * i + 32 * wn, q) : frag(lb, BK, wn * 32 * NB + 32 * i, q);
      }
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
    }
  }
  __syncthreads();

  // Bands of 64 rows through LDS.  Accumulator register r of block (i, j) holds row
  // 8 (r / 4) + 4 h + r % 4, column xl of it.
  float *stage = reinterpret_cast<float *>(lds);
  constexpr int BANDS = TB / BAND;
#pragma unroll
  for (int ps = 0; ps < BANDS; ++ps) {
    if (ps) __syncthreads();
    if (wm == ps * BAND / (32 * NB)) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            // columns of the gate come first, then up's: 32 NB of a wave are 16 NB of each
            const int col = !TWO ? wn * 32 * NB + 32 * j
                                 : (j >= NB / 2 ? TB / 2 : 0) + wn * 16 * NB + 32 * (j % (NB / 2 ? NB / 2 : 1));
            stage[(32 * i + 8 * (r >> 2) + 4 * h + (r & 3)) * SLD + col + xl] = acc[(2 * ps) % NB + i][j][r];
          }
    }
    __syncthreads();
    const int row0 = m0 + BAND * ps;
    if constexpr (EPI == GP_GATED) {
      constexpr int UNITS = TB / 2 / 8;          // of eight columns
#pragma unroll
      for (int v = tid; v < BAND * UNITS; v += GP_THREADS) {
        const int r = v / UNITS, c = 8 * (v % UNITS), row = row0 + r, col = n0 + c;
        if (row >= p.M || col >= p.N) continue;
        v4u og, ou, oh;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint16_t g[2], u[2], o[2];
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const float x = stage[r * SLD + c + 2 * e + w], y = stage[r * SLD + TB / 2 + c + 2 * e + w];
            g[w] = gp_round(x);
            u[w] = gp_round(y);
            o[w] = gp_round(gp_act(x, p.act) * y);
          }
          og[e] = g[0] | (uint32_t)g[1] << 16;
          ou[e] = u[0] | (uint32_t)u[1] << 16;
          oh[e] = o[0] | (uint32_t)o[1] << 16;
        }
        const int64_t at = (int64_t)row * p.ldc + col;
        *reinterpret_cast<v4u *>(static_cast<uint16_t *>(p.C[0]) + at) = oh;
        if (p.keep_gate) {
          *reinterpret_cast<v4u *>(p.keep_gate + at) = og;
          *reinterpret_cast<v4u *>(p.keep_up + at) = ou;
        }
      }
    } else {
      constexpr int UNITS = TB / 8;
#pragma unroll
      for (int v = tid; v < BAND * UNITS; v += GP_THREADS) {
        const int r = v / UNITS, c = 8 * (v % UNITS), row = row0 + r, col = n0 + c;
        if (row >= p.M || col >= p.N) continue;
        const float *x = stage + r * SLD + c;
        const int64_t at = (int64_t)row * p.ldc + col;
        if constexpr (EPI == GP_F32) {
          float *o = static_cast<float *>(p.C[which]) + at;
          *reinterpret_cast<float4 *>(o) = make_float4(x[0], x[1], x[2], x[3]);
          *reinterpret_cast<float4 *>(o + 4) = make_float4(x[4], x[5], x[6], x[7]);
        } else if constexpr (EPI == GP_BF16) {
          v4u o;
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = gp_round(x[2 * e]) | (uint32_t)gp_round(x[2 * e + 1]) << 16;
          *reinterpret_cast<v4u *>(static_cast<uint16_t *>(p.C[which]) + at) = o;
        } else {
          const v4u g = *reinterpret_cast<const v4u *>(p.gate + at), u = *reinterpret_cast<const v4u *>(p.up + at);
          v4u og, ou, oh;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint16_t a[2], b[2], o[2];
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              const float gv = gp_float((uint16_t)(g[e] >> 16 * w)), uv = gp_float((uint16_t)(u[e] >> 16 * w));
              const float d = x[2 * e + w], f = gp_act(gv, p.act);
              a[w] = gp_round(d * uv * gp_dact(gv, p.act));
              b[w] = gp_round(d * f);
              o[w] = gp_round(f * uv);
            }
            og[e] = a[0] | (uint32_t)a[1] << 16;
            ou[e] = b[0] | (uint32_t)b[1] << 16;
            oh[e] = o[0] | (uint32_t)o[1] << 16;
          }
          *reinterpret_cast<v4u *>(static_cast<uint16_t *>(p.C[0]) + at) = og;
          *reinterpret_cast<v4u *>(static_cast<uint16_t *>(p.C[1]) + at) = ou;
          *reinterpret_cast<v4u *>(p.hidden + at) = oh;
        }
      }
    }
  }
}

template <bool AK, bool BK, int EPI>
hipError_t gp_launch(GpParams p, hipStream_t s) {
  constexpr int TB = 128;
  if (p.M <= 0 || p.N <= 0) return hipSuccess;
  p.tiles_m = (p.M + TB - 1) / TB;
  const int width = EPI == GP_GATED ? TB / 2 : TB;
  p.tiles_n = (p.N + width - 1) / width * (p.pairs ? 2 : 1);
  hipLaunchKernelGGL((product_tiles<AK, BK, EPI, 2>), dim3((unsigned)p.tiles_m * p.tiles_n), dim3(GP_THREADS), 0, s, p);
  return hipGetLastError();
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace

size_t gated_workspace_bytes(int64_t tokens, int64_t n, bool backward) {
  return (backward ? 3 : 1) * up256(2 * (size_t)tokens * (size_t)n);
}

hipError_t launch_gated_fwd(const GatedDesc &d, hipStream_t s) {
  if (d.tokens <= 0) return hipSuccess;
  uint16_t *hidden = static_cast<uint16_t *>(d.workspace);
  GpParams p{};
  p.M = (int)d.tokens; p.N = (int)d.n; p.K = (int)d.m; p.segments = 1;
  p.A[0] = d.x; p.lda = d.ldx; p.B[0] = d.w_gate; p.B[1] = d.w_up; p.ldb = d.n;
  p.C[0] = hidden; p.ldc = d.n; p.keep_gate = d.gate; p.keep_up = d.up; p.act = d.act;
  hipError_t e = gp_launch<true, false, GP_GATED>(p, s);
  if (e != hipSuccess) return e;
  p = GpParams{};
  p.M = (int)d.tokens; p.N = (int)d.p; p.K = (int)d.n; p.segments = 1;
  p.A[0] = hidden; p.lda = d.n; p.B[0] = d.w_down; p.ldb = d.p;
  p.C[0] = d.y; p.ldc = d.ldy;
  return gp_launch<true, false, GP_BF16>(p, s);
}

hipError_t launch_gated_bwd(const GatedDesc &d, hipStream_t s) {
  const size_t each = up256(2 * (size_t)d.tokens * (size_t)d.n);
  char *w = static_cast<char *>(d.workspace);
  uint16_t *dg = (uint16_t *)w, *du = (uint16_t *)(w + each), *hidden = (uint16_t *)(w + 2 * each);
  hipError_t e = hipSuccess;
  GpParams p{};
  if (d.tokens > 0) {
    p.M = (int)d.tokens; p.N = (int)d.n; p.K = (int)d.p; p.segments = 1;
    p.A[0] = d.dy; p.lda = d.lddy; p.B[0] = d.w_down; p.ldb = d.p;
    p.C[0] = dg; p.C[1] = du; p.hidden = hidden; p.ldc = d.n; p.gate = d.gate; p.up = d.up; p.act = d.act;
    if ((e = gp_launch<true, true, GP_DGATED>(p, s)) != hipSuccess) return e;
    if (d.dx) {
      p = GpParams{};
      p.M = (int)d.tokens; p.N = (int)d.m; p.K = (int)d.n; p.segments = 2;
      p.A[0] = dg; p.A[1] = du; p.lda = d.n; p.B[0] = d.w_gate; p.B[1] = d.w_up; p.ldb = d.n;
      p.C[0] = d.dx; p.ldc = d.lddx;
      if ((e = gp_launch<true, true, GP_BF16>(p, s)) != hipSuccess) return e;
    }
  }
  auto grad = [&](const GpParams &q) {
    return d.grad_bf16 ? gp_launch<false, false, GP_BF16>(q, s) : gp_launch<false, false, GP_F32>(q, s);
  };
  if (d.dw_gate || d.dw_up) {
    p = GpParams{};
    p.M = (int)d.m; p.N = (int)d.n; p.K = (int)d.tokens; p.segments = 1;
    p.A[0] = d.x; p.lda = d.ldx; p.ldb = d.n; p.ldc = d.n;
    p.pairs = d.dw_gate && d.dw_up;
    p.B[0] = d.dw_gate ? dg : du; p.B[1] = du; p.C[0] = d.dw_gate ? d.dw_gate : d.dw_up; p.C[1] = d.dw_up;
    if ((e = grad(p)) != hipSuccess) return e;
  }
  if (d.dw_down) {
    p = GpParams{};
    p.M = (int)d.n; p.N = (int)d.p; p.K = (int)d.tokens; p.segments = 1;
    p.A[0] = hidden; p.lda = d.n; p.B[0] = d.dy; p.ldb = d.lddy; p.C[0] = d.dw_down; p.ldc = d.p;
    if ((e = grad(p)) != hipSuccess) return e;
  }
  return e;
}

}  // namespace soap
