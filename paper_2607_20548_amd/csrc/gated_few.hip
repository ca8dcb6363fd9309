// Products of few rows for the gated feed-forward block: Y = X W over up to 64 tokens, bound by
// reading the weights once.
//
// A workgroup takes 64 columns (of both the gate's and up's weights forward) and a part of k,
// its four waves a quarter of that each.  A wave loads slabs of 32 k, weights and
// tokens, through a ring of its own in LDS and waits for nobody: 30 to 36 KB of each are in flight
// while it multiplies the oldest, 120 to 144 KB for a compute unit.  Weights come as they lie
// (x-contiguous rows of k, read transposed, or k-contiguous rows), the matrix instructions take
// them as rows and 32 tokens as columns.  The waves' sums meet in LDS, in their order, and go
// through the activation or its gradient, or are rounded, there, or where columns are few and k
// has parts, are written as fp32 sums that a second kernel adds in their order.
//
// H forward and dG, dU and H backward are kept in two bfloat16 halves (their rounding and what that
// leaves), which costs matrix instructions that the weights' loads cover, and no bytes to speak of:
// of few roundings the largest would show in a result (six tokens' dX: 1.5 times the error of
// its own rounding alone).
#include "products_bf16.h"

#include <algorithm>

namespace soap {
namespace {

// Bytes of a product's weights from which they are loaded past the caches (16 x 4096 x 14336 forward 82.8 and
// 79.1 us, 12 x 2048 x 8192 backward 89.2 and 82.1; 24 x 1000 x 3000 forward 23.4 and 31.3).
constexpr int64_t GF_CACHED = 60 << 20;
constexpr int GF_KB = 32, GF_COLS = 64;
constexpr int GF_W = GF_KB * GF_COLS * 2, GF_X = 32 * GF_KB * 2;   // bytes of a slab's weights, of 32 tokens

struct GfParams {
  int T, N, K;                   // K: of a segment
  const uint16_t *X[4], *W[2];   // X by segment and half; W by segment, or gate's and up's
  int64_t ldx, ldw;
  int segments, splits, chunks, far;
  float *part;                   // [split][matrix][T][N]
  GatedJoin out;                 // of a product in one part
};

// ------------------------------------------------- what is made of the sums
enum { GJ_PART, GJ_GATED, GJ_DGATED, GJ_BF16, GJ_F32 };

// Two values' rounding, and what it leaves, rounded: the lower halves.  An infinity leaves nothing; a
// finite value past bfloat16's largest is that and a remainder.
struct GjHalves {
  uint32_t high, low;
};
__device__ __forceinline__ GjHalves gj_halves(const float (&v)[2]) {
  uint32_t h[2];
  float l[2];
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    h[w] = gp_round(v[w]);
    const bool past = (h[w] & 0x7fffu) == 0x7f80u, inf = fabsf(v[w]) == INFINITY;
    h[w] -= past && !inf;
    l[w] = inf ? 0.f : v[w] - gp_float((uint16_t)h[w]);
  }
  return {h[0] | h[1] << 16, gp_pack(l[0], l[1])};
}

// Of eight columns of a row: x[0], and x[1] of up's.
template <int MODE, int ACT>
__device__ __forceinline__ void gj_finish(const GatedJoin &p, const float (*x)[8], int64_t row, int64_t col) {
  const int64_t at = row * p.N + col;
  if constexpr (MODE == GJ_BF16) {
    v4u o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = gp_pack(x[0][2 * e], x[0][2 * e + 1]);
    *reinterpret_cast<v4u *>(p.out + row * p.ldo + col) = o;
  } else if constexpr (MODE == GJ_F32) {
    float *o = p.out_f32 + row * p.ldo + col;
    *reinterpret_cast<float4 *>(o) = make_float4(x[0][0], x[0][1], x[0][2], x[0][3]);
    *reinterpret_cast<float4 *>(o + 4) = make_float4(x[0][4], x[0][5], x[0][6], x[0][7]);
  } else if constexpr (MODE == GJ_GATED) {
    v4u og, ou, oh, ol;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float hv[2];
#pragma unroll
      for (int w = 0; w < 2; ++w) hv[w] = gp_act<ACT>(x[0][2 * e + w]).a * x[1][2 * e + w];
      og[e] = gp_pack(x[0][2 * e], x[0][2 * e + 1]);
      ou[e] = gp_pack(x[1][2 * e], x[1][2 * e + 1]);
      oh[e] = gp_pack(hv[0], hv[1]);
      if (p.low) {
        const GjHalves r = gj_halves(hv);
        oh[e] = r.high;
        ol[e] = r.low;
      }
    }
    *reinterpret_cast<v4u *>(p.out + at) = oh;
    if (p.low) *reinterpret_cast<v4u *>(p.low + at) = ol;
    if (p.keep_gate) {
      *reinterpret_cast<v4u *>(p.keep_gate + at) = og;
      *reinterpret_cast<v4u *>(p.keep_up + at) = ou;
    }
  } else {
    const v4u g = *reinterpret_cast<const v4u *>(p.gate + at), u = *reinterpret_cast<const v4u *>(p.up + at);
    v4u og, ou, oh, lg, lu, lh;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float a[2], b[2], o[2];
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const float uv = gp_float((uint16_t)(u[e] >> 16 * w)), d = x[0][2 * e + w];
        const GpAct f = gp_act<ACT>(gp_float((uint16_t)(g[e] >> 16 * w)));
        a[w] = d * uv * f.d;
        b[w] = d * f.a;
        o[w] = f.a * uv;
      }
      og[e] = gp_pack(a[0], a[1]);
      ou[e] = gp_pack(b[0], b[1]);
      oh[e] = gp_pack(o[0], o[1]);
      if (p.low) {
        const GjHalves ra = gj_halves(a), rb = gj_halves(b), ro = gj_halves(o);
        og[e] = ra.high;
        lg[e] = ra.low;
        ou[e] = rb.high;
        lu[e] = rb.low;
        oh[e] = ro.high;
        lh[e] = ro.low;
      }
    }
    *reinterpret_cast<v4u *>(p.out + at) = og;
    *reinterpret_cast<v4u *>(p.out2 + at) = ou;
    *reinterpret_cast<v4u *>(p.hidden + at) = oh;
    if (p.low) {
      *reinterpret_cast<v4u *>(p.low + at) = lg;
      *reinterpret_cast<v4u *>(p.low2 + at) = lu;
      *reinterpret_cast<v4u *>(p.hidden_low + at) = lh;
    }
  }
}

// WK: weights k-contiguous.  TWO: gate's and up's.  NX: halves of X.  RB: 32s of tokens.
template <bool WK, bool TWO, int NX, int RB>
struct GfShape {
  static constexpr int M = TWO ? 2 : 1, WB = M * GF_W, XB = NX * RB * GF_X, SLAB = WB + XB;
  static constexpr int RING = 40960 / SLAB > 5 ? 5 : 40960 / SLAB;
  static constexpr int LOADS = SLAB / 1024;
};

// FIN: what is made of the sums (GJ_PART: they are written as they are).  FAR: weights loaded past the
// caches.
template <bool WK, bool TWO, int NX, int RB, int FIN, int ACT, bool FAR>
__global__ __launch_bounds__(GP_THREADS, 1) void product_few(GfParams p) {
  using S = GfShape<WK, TWO, NX, RB>;
  constexpr int M = S::M, RING = S::RING;
  constexpr int SLD = M * GF_COLS + 4;                     // row of the waves' sums, floats
  static_assert(4 * 32 * SLD * 4 <= 4 * RING * S::SLAB, "the sums fit the rings");
  static_assert((RING - 1) * S::LOADS <= 63, "the counter of loads");
  __shared__ __attribute__((aligned(1024))) uint8_t lds[4 * RING * S::SLAB];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int xl = lane & 31, h = lane >> 5;
  const int chunk = blockIdx.x % p.chunks, z = blockIdx.x / p.chunks, n0 = chunk * GF_COLS;
  const int64_t ldx2 = 2 * p.ldx, ldw2 = 2 * p.ldw;
  uint8_t *mine = lds + wave * RING * S::SLAB;
  const uint32_t base = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)mine);

  // a load's lane -> row and unit of 16 bytes, permuted so that a read's lanes meet in no bank
  const int rk = lane >> 2, uk = (lane & 3) ^ ((lane >> 4) & 3);         // k-contiguous: rows of 64 bytes
  const int rx = lane >> 3, ux = (lane & 7) ^ (4 * ((lane >> 4) & 1));   // x-contiguous: of 128
  const uint32_t offw = WK ? (uint32_t)(rk * ldw2) + 16 * uk : (uint32_t)(rx * ldw2) + 16 * ux;
  const uint32_t offx = (uint32_t)(rk * ldx2) + 16 * uk;
  const int nk1 = (p.K + GF_KB - 1) / GF_KB;
  const int64_t nk = (int64_t)nk1 * p.segments;
  const int first = (int)((z * 4 + wave) * nk / (4 * p.splits)), last = (int)((z * 4 + wave + 1) * nk / (4 * p.splits));

  auto issue = [&](int s) {                                // slab s, or nothing in its place past the last
    const bool live = s < last;
    const int seg = p.segments > 1 && s >= nk1, at = s - (seg ? nk1 : 0), left = p.K - at * GF_KB;
    const uint32_t to = base + (uint32_t)((s - first) % RING) * S::SLAB;
    const uint32_t dead = 8 * uk >= left ? GP_OUT : 0u;    // a unit past the end of k
#pragma unroll
    for (int t = 0; t < M; ++t) {
      GpSource w;
      w.start(TWO ? p.W[t] : p.W[seg], WK, n0, p.N, p.K, ldw2, GF_KB);
      w.next(at);
      if (!live) w.left = 0;
      const v4i r = w.buffer();
#pragma unroll
      for (int i = 0; i < 4; ++i)
        gp_load<FAR>(r, to + t * GF_W + 1024 * i, (offw + (uint32_t)((WK ? 16 : 8) * i * ldw2)) | (WK ? dead : 0u));
    }
#pragma unroll
    for (int t = 0; t < NX; ++t) {
      GpSource x;
      x.start(p.X[2 * seg + t], true, 0, p.T, p.K, ldx2, GF_KB);
      x.next(at);
      if (!live) x.left = 0;
      const v4i r = x.buffer();
#pragma unroll
      for (int i = 0; i < 2 * RB; ++i)
        gp_load(r, to + S::WB + t * RB * GF_X + 1024 * i, (offx + (uint32_t)(16 * i * ldx2)) | dead);
    }
  };

  v16f acc[M][2][RB];
#pragma unroll
  for (int t = 0; t < M; ++t)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[t][j][b][r] = 0.f;

#pragma unroll
  for (int s = 0; s < RING; ++s) issue(first + s);
  const int i16 = lane & 15, r4 = i16 >> 2, u0 = 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1);
  for (int s = first; s < last; ++s) {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((RING - 1) * S::LOADS) : "memory");
    const uint8_t *w = mine + (s - first) % RING * S::SLAB, *x = w + S::WB;
    v8bf fw[2][M][2], fx[2][NX][RB];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
#pragma unroll
      for (int t = 0; t < M; ++t)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (WK) fw[q][t][j] = *reinterpret_cast<const v8bf *>(w + t * GF_W + (32 * j + xl) * 64 + 16 * ((2 * q + h) ^ ((xl >> 2) & 3)));
          else fw[q][t][j] = gp_read_transposed(w + t * GF_W + (16 * q + 8 * h + r4) * 128 + 16 * ((4 * j + u0) ^ (4 * (r4 >> 1))) + 8 * (i16 & 1), 128);
        }
#pragma unroll
      for (int t = 0; t < NX; ++t)
#pragma unroll
        for (int b = 0; b < RB; ++b)
          fx[q][t][b] = *reinterpret_cast<const v8bf *>(x + (t * RB + b) * GF_X + xl * 64 + 16 * ((2 * q + h) ^ ((xl >> 2) & 3)));
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // read: the place is free
    issue(s + RING);
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int v = 0; v < NX; ++v)
#pragma unroll
        for (int t = 0; t < M; ++t)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int b = 0; b < RB; ++b)
              acc[t][j][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fw[q][t][j], fx[q][v][b], acc[t][j][b], 0, 0, 0);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

  // register r of a block: column 8 (r / 4) + 4 h + r % 4 of the weights, token xl
  float *stage = reinterpret_cast<float *>(lds);
  constexpr int UNITS = GF_COLS / 8;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    __syncthreads();
#pragma unroll
    for (int t = 0; t < M; ++t)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          *reinterpret_cast<float4 *>(stage + (wave * 32 + xl) * SLD + t * GF_COLS + 32 * j + 2 * r + 4 * h) =
              make_float4(acc[t][j][b][r], acc[t][j][b][r + 1], acc[t][j][b][r + 2], acc[t][j][b][r + 3]);
    __syncthreads();
    const int c = 8 * (tid % UNITS), token = 32 * b + tid / UNITS, n = n0 + c;   // 32 rows of 8 units
    if (token >= p.T || n >= p.N) continue;
    float o[M][8];
#pragma unroll
    for (int t = 0; t < M; ++t)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float *x = stage + tid / UNITS * SLD + t * GF_COLS + c + e;
        o[t][e] = x[0];
#pragma unroll
        for (int w = 1; w < 4; ++w) o[t][e] += x[w * 32 * SLD];
      }
    if constexpr (FIN == GJ_PART) {
#pragma unroll
      for (int t = 0; t < M; ++t) {
        float *to = p.part + (((int64_t)z * M + t) * p.T + token) * p.N + n;
        *reinterpret_cast<float4 *>(to) = make_float4(o[t][0], o[t][1], o[t][2], o[t][3]);
        *reinterpret_cast<float4 *>(to + 4) = make_float4(o[t][4], o[t][5], o[t][6], o[t][7]);
      }
    } else {
      gj_finish<FIN, ACT>(p.out, o, token, n);
    }
  }
}

// ------------------------------------------------- the parts' sums
constexpr int GJ_THREADS = 256;

// Eight columns of a row a thread.
template <int MODE, int ACT>
__global__ __launch_bounds__(GJ_THREADS) void product_join(GatedJoin p) {
  const int64_t units = p.N / 8, i = (int64_t)blockIdx.x * GJ_THREADS + threadIdx.x;
  if (i >= p.T * units) return;
  const int64_t row = i / units, col = 8 * (i - row * units), at = row * p.N + col, size = p.T * p.N;
  constexpr int M = MODE == GJ_GATED ? 2 : 1;
  float x[M][8];
#pragma unroll
  for (int t = 0; t < M; ++t) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[t][e] = 0.f;
    for (int z = 0; z < p.splits; ++z) {
      const float4 *q = reinterpret_cast<const float4 *>(p.part + (z * M + t) * size + at);
      const float4 a = q[0], b = q[1];
      x[t][0] += a.x; x[t][1] += a.y; x[t][2] += a.z; x[t][3] += a.w;
      x[t][4] += b.x; x[t][5] += b.y; x[t][6] += b.z; x[t][7] += b.w;
    }
  }
  gj_finish<MODE, ACT>(p, x, row, col);
}

template <int MODE, int ACT>
hipError_t gj_launch(const GatedJoin &p, hipStream_t s) {
  const int64_t n = p.T * (p.N / 8);
  hipLaunchKernelGGL((product_join<MODE, ACT>), dim3((unsigned)((n + GJ_THREADS - 1) / GJ_THREADS)), dim3(GJ_THREADS), 0, s, p);
  return hipGetLastError();
}

template <bool WK, bool TWO, int NX, int FIN, int ACT = 0>
hipError_t gf_launch(const GfParams &p, hipStream_t s) {
  const dim3 grid((unsigned)(p.chunks * p.splits)), block(GP_THREADS);
#define SOAP_FEW(RB, FAR) hipLaunchKernelGGL((product_few<WK, TWO, NX, RB, FIN, ACT, FAR>), grid, block, 0, s, p)
  if (p.T <= 32) { if (p.far) SOAP_FEW(1, true); else SOAP_FEW(1, false); }
  else { if (p.far) SOAP_FEW(2, true); else SOAP_FEW(2, false); }
#undef SOAP_FEW
  return hipGetLastError();
}

}  // namespace

hipError_t launch_gated_join(const GatedJoin &p, hipStream_t s) {
  if (p.kind == GatedJoin::BF16) return gj_launch<GJ_BF16, 0>(p, s);
  if (p.kind == GatedJoin::F32) return gj_launch<GJ_F32, 0>(p, s);
  if (p.kind == GatedJoin::GATED)
    return p.act == SOAP_ACT_SILU ? gj_launch<GJ_GATED, SOAP_ACT_SILU>(p, s) : gj_launch<GJ_GATED, SOAP_ACT_GELU>(p, s);
  return p.act == SOAP_ACT_SILU ? gj_launch<GJ_DGATED, SOAP_ACT_SILU>(p, s) : gj_launch<GJ_DGATED, SOAP_ACT_GELU>(p, s);
}

// Parts of k: as many as give compute units a workgroup each and none a second, of six slabs a
// wave at least (4096 x 14336, 16 tokens: 224 workgroups for the columns alone 83 us, 448 93; one
// token of 512 x 1024: parts of two slabs 20.0, of four 17.1, of six 14.4, of eight 14.5; 64 of
// 1000 x 3000: 30.0, 27.9, 29.7 and 33.4).
int few_splits(int64_t N, int64_t slabs) {
  const int64_t chunks = (N + GF_COLS - 1) / GF_COLS;
  return (int)std::max<int64_t>(1, std::min(256 / chunks, slabs / 24));
}

// The product, and what is made of it.
hipError_t launch_product_few(const FewDesc &d, const GatedJoin &out, hipStream_t s) {
  GfParams p{};
  p.T = (int)d.tokens; p.N = (int)d.n; p.K = (int)d.k;
  p.W[0] = d.w[0]; p.W[1] = d.w[1]; p.ldx = d.ldx; p.ldw = d.ldw;
  for (int i = 0; i < 4; ++i) p.X[i] = d.x[i];
  p.segments = d.segments; p.chunks = (p.N + GF_COLS - 1) / GF_COLS; p.part = d.part;
  p.splits = few_splits(d.n, (d.k + GF_KB - 1) / GF_KB * d.segments);
  p.far = 2 * d.k * d.segments * d.n * (d.kind == FewDesc::GATE_UP ? 2 : 1) > GF_CACHED;
  p.out = out;
  p.out.T = d.tokens; p.out.N = d.n; p.out.part = d.part; p.out.splits = p.splits;
  const bool silu = out.act == SOAP_ACT_SILU;
  hipError_t e;
  if (p.splits == 1) {
    if (d.kind == FewDesc::GATE_UP)
      return silu ? gf_launch<false, true, 1, GJ_GATED, SOAP_ACT_SILU>(p, s) : gf_launch<false, true, 1, GJ_GATED, SOAP_ACT_GELU>(p, s);
    if (d.kind == FewDesc::HALVES) return gf_launch<false, false, 2, GJ_BF16>(p, s);
    if (d.kind == FewDesc::ROWS_HALVES) return gf_launch<true, false, 2, GJ_BF16>(p, s);
    return silu ? gf_launch<true, false, 1, GJ_DGATED, SOAP_ACT_SILU>(p, s) : gf_launch<true, false, 1, GJ_DGATED, SOAP_ACT_GELU>(p, s);
  }
  if (d.kind == FewDesc::GATE_UP) e = gf_launch<false, true, 1, GJ_PART>(p, s);
  else if (d.kind == FewDesc::HALVES) e = gf_launch<false, false, 2, GJ_PART>(p, s);
  else if (d.kind == FewDesc::ROWS_HALVES) e = gf_launch<true, false, 2, GJ_PART>(p, s);
  else e = gf_launch<true, false, 1, GJ_PART>(p, s);
  return e != hipSuccess ? e : launch_gated_join(p.out, s);
}

}  // namespace soap
