// The gated feed-forward block and its gradients in bfloat16, sums in fp32:
//
//   G = X Wg,  U = X Wu,  H = act(G) * U,  Y = H Wd
//   dH = dY Wd^T,  dG = dH * U * act'(G),  dU = dH * act(G)
//   dX = dG Wg^T + dU Wu^T,  dWg = X^T dG,  dWu = X^T dU,  dWd = H^T dY
//
// X is tokens x m, Wg and Wu m x n, Wd n x p.  H, dG and dU are rounded to bfloat16 once, as
// the operands of the next product (of up to 64 tokens to two bfloat16, whose products are added);
// act works on fp32 sums forward and on the kept (rounded) G and U backward.  That one rounding makes the
// error of Y, dX and the weights' gradients sqrt 2 times that of their own rounding.  Two bfloat16 for more
// tokens too would take it away, and double the matrix instructions behind them: 8192 x 2048 x 8192 forward 694
// us and 884, backward 1349 and 2324, before the lower halves' own bytes; 300 x 4096 x 8192 93 and 117, 192 and
// 288.  Up to 64 tokens the weights' loads hide them.
//
// Products of up to 64 tokens are product_few's; all others are one kernel's, product_tiles: C =
// sum over k of A(x, k) B(y, k), its operands in memory either k-contiguous ([x][k]: X, H, dY,
// dG, dU, and the weights seen from their rows) or x-contiguous ([k][x]: the weights forward, and
// both operands of the weights' gradients), so that nothing is transposed beforehand.  Both come to
// LDS as they are in memory, by loads that write LDS themselves, in blocks of 64 rows of 128
// bytes, 16-byte units permuted within a row so that no two of a read's lanes meet in a bank:
// k-contiguous blocks are read 16 bytes of a row at a time, x-contiguous ones by the transposing
// reads, which give a lane four k of its own x.
//
// What bounds it, 8192 x 2048 x 8192: matrix instructions where sums are long (dX 405 us, 1355 TFLOP/s,
// busy 0.79 of the cycles; the weights' gradients 614, 1340), and where an activation is behind
// them, the outputs that all compute units write at the same time (H, G and U 498; dG, dU and
// H from G and U 368, of which 246 without their bytes).  The whole: 702 to 715 forward (1165
// TFLOP/s), 1379 to 1400 backward (1185), with fp32 gradients of weights 1430.
//
// Operands past their ends read as zeros (buffer bounds; units past the end of k are sent
// out of bounds), so that sizes need no multiple of a tile; m, n and p are multiples of 8
// and rows 16-byte aligned, so that no unit crosses an end.
#include "products_bf16.h"

#include <algorithm>
#include <type_traits>

namespace soap {
namespace {

constexpr int GP_KB = 64;                        // k of a slab
// Bytes of weights' gradients from which they are stored past the caches, if they are bfloat16 (100 x 2048 x 8192:
// 96.8 and 87.2 us, 777 x 1160 x 2744: 78.8 and 77.4, 1 x 512 x 1024: 24.0 and 27.7).  Not fp32, of which
// a lane stores 16 bytes of every 32 at a time: past the caches 12 x 2048 x 8192 151 us, through them 93; 300 x
// 4096 x 8192 473 and 260, 8192 x 2048 x 8192 1476 and 1433.
constexpr int64_t GP_CACHED = 16 << 20;
static_assert(GP_CACHED >= 2 * 256 * 128 * 128, "more than 256 tiles of 128 past the caches");
constexpr int GP_BLOCK = 64 * 128;               // bytes of a block of 64 rows in LDS

enum { GP_BF16, GP_F32, GP_GATED, GP_DGATED, GP_PART, GP_BF16_FAR };

struct GpOther {               // product over the same k
  int M, N, tiles_m, tiles_n;
  const uint16_t *A[2], *B[2];
  void *C;
  int64_t lda, ldb, ldc;
};

struct GpParams {
  int M, N, K;                 // N: of one matrix; K: of one segment
  const uint16_t *A[2], *B[2]; // [1]: up's weights, or the second segment of k
  int64_t lda, ldb;
  int segments;                // of k, each with operands of its own
  int splits;                  // parts of k, the grid's y; more than one write fp32 sums
  int tiles_m, tiles_n;
  int others;                  // of the weights' gradients: one launch takes all three
  GpOther other[2];
  void *C[2];                  // part: [part][matrix][M][N] floats
  int64_t ldc;
  // gated: C[0] the product, kept G and U (or null); dgated: C[0] = dG, C[1] = dU, H
  const uint16_t *gate, *up;
  uint16_t *keep_gate, *keep_up, *hidden;
};

// NB: blocks of 32 x 32 on a side of a wave's share; tiles of 64 NB.  ACT: of the epilogues
// with an activation.  TWO: columns of both gate and up.  RING: operands' slabs in LDS (odd).
template <bool AK, bool BK, int EPI, int NB, int ACT, bool TWO, int RING>
__global__ __launch_bounds__(GP_THREADS, NB == 4 || RING > 5 ? 1 : 2) void product_tiles(GpParams p) {
  constexpr int TB = 64 * NB, SUB = TB / 64, OP = SUB * GP_BLOCK, LOADS = 2 * SUB;
  constexpr int SLD = TB + 4;                    // staging row of the epilogue, floats
  constexpr int BAND = 64;
  static_assert(2 * BAND * SLD * 4 <= RING * OP, "two of the epilogue's bands fit the ring");
  __shared__ __attribute__((aligned(1024))) uint8_t lds[RING * OP];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1, xl = lane & 31, h = lane >> 5;

  // the tile: a contiguous run for each XCD, eight tiles of rows by all columns at a time
  int tm, tn;
  {
    const int nt = gridDim.x, q = nt >> 3, r = nt & 7, x = blockIdx.x & 7;
    int t = x * q + min(x, r) + (blockIdx.x >> 3);
    if constexpr (!AK && !BK) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (i < p.others && t >= p.tiles_m * p.tiles_n) {
          t -= p.tiles_m * p.tiles_n;
          const GpOther o = p.other[i];
          p.M = o.M; p.N = o.N; p.tiles_m = o.tiles_m; p.tiles_n = o.tiles_n;
          p.A[0] = o.A[0]; p.A[1] = o.A[1]; p.B[0] = o.B[0]; p.B[1] = o.B[1]; p.C[0] = o.C; p.lda = o.lda; p.ldb = o.ldb; p.ldc = o.ldc;
        } else {
          break;
        }
    }
    const int group = t / (8 * p.tiles_n), first = 8 * group, size = min(p.tiles_m - first, 8);
    const int in = t - group * 8 * p.tiles_n;
    tm = __builtin_amdgcn_readfirstlane(first + in % size);
    tn = __builtin_amdgcn_readfirstlane(in / size);
  }
  const int m0 = tm * TB, n0 = tn * (TWO ? TB / 2 : TB);
  const int64_t lda2 = 2 * p.lda, ldb2 = 2 * p.ldb;

  // a wave's loads: of block j >> 3 the rows 8 (j & 7) .., j = wave + 4 i
  uint32_t offa[LOADS], offb[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int j = wave + 4 * i, s = j >> 3, row = 8 * (j & 7) + (lane >> 3);
    const int uk = (lane & 7) ^ ((row >> 1) & 7), ux = (lane & 7) ^ (4 * ((row >> 1) & 1));
    offa[i] = AK ? (uint32_t)((64 * s + row) * lda2) + 16 * uk : (uint32_t)(row * lda2) + 128 * s + 16 * ux;
    const int sb = TWO ? s >> 1 : s;
    offb[i] = BK ? (uint32_t)((64 * sb + row) * ldb2) + 16 * uk : (uint32_t)(row * ldb2) + 128 * sb + 16 * ux;
  }
  // the unit of eight k that a lane loads, the same in all its rows
  const int unit = (lane & 7) ^ ((4 * (wave & 1) + (lane >> 4)) & 7);
  const uint32_t base = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds);
  const int nk1 = (p.K + GP_KB - 1) / GP_KB, all = nk1 * p.segments;
  const int s0 = (int)((int64_t)blockIdx.y * all / p.splits), nk = (int)((int64_t)(blockIdx.y + 1) * all / p.splits) - s0;

  // A slab of A and one of B take a place each of a ring, in the order A0 B0 A1 B1 ..: of five, what
  // slab k frees takes B of slab k + 2, which then has a slab's time to arrive, and A of slab k + 3,
  // which has two; of nine, two slabs more.
  struct Stream {
    GpSource s0, s1;
    v4i r0, r1;
    int left, slab, place;                       // of k in the segment; the next slab; its place
    uint32_t dead, to;
  } sa, sb;
  sa.slab = sb.slab = s0;
  sa.place = 0;
  sb.place = 1;
  auto begin = [&](Stream &s, bool is_a) {       // the next slab of an operand: its loads may follow
    if (s.slab == s0 || (p.segments > 1 && s.slab == nk1)) {
      const int seg = p.segments > 1 && s.slab >= nk1, at = s.slab - (seg ? nk1 : 0);
      if (is_a) s.s0.start(p.A[seg], AK, m0, p.M, p.K, lda2, GP_KB);
      else s.s0.start(p.B[seg], BK, n0, p.N, p.K, ldb2, GP_KB);
      if (TWO && !is_a) s.s1.start(p.B[1], BK, n0, p.N, p.K, ldb2, GP_KB);
      s.s0.next(at);
      if (TWO && !is_a) s.s1.next(at);
      s.left = p.K - at * GP_KB;
    }
    s.r0 = s.s0.buffer();
    if (TWO && !is_a) s.r1 = s.s1.buffer();
    s.dead = 8 * unit >= s.left ? GP_OUT : 0u;   // a unit past the end of k
    s.to = base + s.place * OP + wave * 1024;
    s.s0.next();
    if (TWO && !is_a) s.s1.next();
    s.left -= GP_KB;
    ++s.slab;
    s.place = s.place >= RING - 2 ? s.place - (RING - 2) : s.place + 2;
  };
  auto load = [&](bool is_a, int i) {
    if (is_a) gp_load(sa.r0, sa.to + 4096 * i, AK ? offa[i] | sa.dead : offa[i]);
    else gp_load(TWO && (i >> 1 & 1) ? sb.r1 : sb.r0, sb.to + 4096 * i, BK ? offb[i] | sb.dead : offb[i]);
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
    return gp_read_transposed(at, 128);
  };

  // The epilogue's bands of 64 rows: a thread's units of eight columns, GP_THREADS apart.
  constexpr int UNITS = (EPI == GP_GATED ? TB / 2 : TB) / 8, EACH = BAND * UNITS / GP_THREADS;
  float *stage = reinterpret_cast<float *>(lds);
  const int c = 8 * (tid % UNITS);               // GP_THREADS is a multiple of UNITS
  const int second = EPI == GP_PART && TWO && c >= TB / 2, col = n0 + c - (second ? TB / 2 : 0);
  auto row_of = [&](int ps, int v) {
    const int r = (tid + GP_THREADS * v) / UNITS;
    return m0 + (r >> 5) * 32 * NB + 32 * ps + (r & 31);
  };
  // G and U of two bands, loaded during the first slab, and two bands ahead from then on: before
  // a band's stores, which they would otherwise wait for, one counter counting both (8192 x 8192,
  // K = 2048: one band ahead, behind the stores, 429 us)
  v4u kg[2][EPI == GP_DGATED ? EACH : 1], ku[2][EPI == GP_DGATED ? EACH : 1];
  auto kept = [&](int set, int ps, int v) {
    const int row = row_of(ps, v);
    if (row >= p.M || col >= p.N) return;
    const int64_t at = (int64_t)row * p.ldc + col;
    kg[set][v] = *reinterpret_cast<const v4u *>(p.gate + at);
    ku[set][v] = *reinterpret_cast<const v4u *>(p.up + at);
  };

  v16f acc[NB][NB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  v8bf fa[2][NB], fb[2][NB];
  const uint8_t *la = lds, *lb = lds + OP;       // the slab that is read
  auto read = [&](int f, int q, int u) {         // the u-th of a step's 2 NB fragments
    const int i = u >> 1;
    if (!(u & 1)) fa[f][i] = frag(la, AK, wm * 32 * NB + 32 * i, q);
    // gated: a wave's columns are half the gate's, in even blocks, and half up's
    else fb[f][i] = TWO && NB == 2 ? frag(lb, BK, 64 * i + 32 * wn, q) : frag(lb, BK, wn * 32 * NB + 32 * i, q);
  };
  // One step's matrix instructions, on fragments f, with the reads of the next step's (of step q) and
  // the loads l0 .. l1, of B then of A, spread among them.
  auto step = [&](int f, int q, int l0, int l1) {
    constexpr int MM = NB * NB, RD = 3 * MM / 4;
#pragma unroll
    for (int u = 0; u < MM; ++u) {
#pragma unroll
      for (int v = min(u, RD) * 2 * NB / RD; v < min(u + 1, RD) * 2 * NB / RD; ++v) read(f ^ 1, q, v);
#pragma unroll
      for (int v = l0 + u * (l1 - l0) / MM; v < l0 + (u + 1) * (l1 - l0) / MM; ++v) load(v >= LOADS, v % LOADS);
      acc[u / NB][u % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[f][u % NB], fa[f][u / NB], acc[u / NB][u % NB], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // All but a wave's last `flying` loads, and its reads, then all waves'.
#define GP_ARRIVED(flying)                                                                                \
  do {                                                                                                    \
    __builtin_amdgcn_sched_barrier(0);                                                                    \
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(flying) : "memory"); /* LDS changed */ \
    __builtin_amdgcn_sched_barrier(0);                                                                    \
  } while (0)
  // Loads are spread over the four steps from the barrier that frees their places on: the memory
  // pipe takes 27 cycles for a wave's, all of a step's 512 for five from each of four waves, and
  // one that it does not take yet holds its wave's matrix instructions up.
  constexpr int L1 = 2 * LOADS * 5 / 16, L2 = 2 * LOADS * 10 / 16, L3 = 2 * LOADS * 13 / 16;
#pragma unroll
  for (int u = 0; u < RING - 2; ++u) {           // A0, B0, A1
    if (u & 1) begin(sb, false);
    else begin(sa, true);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load(!(u & 1), i);
  }
  begin(sb, false);
  begin(sa, true);
#pragma unroll
  for (int v = 0; v < L1; ++v) load(v >= LOADS, v % LOADS);
  GP_ARRIVED((RING - 4) * LOADS + L1);
  if constexpr (EPI == GP_DGATED) {
#pragma unroll
    for (int v = 0; v < 2 * EACH; ++v) kept(v / EACH, v / EACH, v % EACH);
  }
#pragma unroll
  for (int u = 0; u < 2 * NB; ++u) read(0, 0, u);
  int pa = 0;                                    // the place of A's slab
  for (int kt = 0; kt < nk; ++kt) {
    __builtin_amdgcn_sched_barrier(0);
    step(0, 1, L1, L2);
    step(1, 2, L2, L3);
    step(0, 3, L3, 2 * LOADS);
    GP_ARRIVED((RING - 4) * LOADS);
    begin(sb, false);
    begin(sa, true);
    pa = pa >= RING - 2 ? pa - (RING - 2) : pa + 2;
    la = lds + pa * OP;
    lb = pa == RING - 1 ? lds : la + OP;
    step(1, 0, 0, L1);
  }
  GP_ARRIVED(0);

  // Bands of 64 rows, 32 of either half of the tile, through LDS.  B's values came first in the
  // matrix instructions: register r of block (i, j) holds row xl of A's, column
  // 8 (r / 4) + 4 h + r % 4 of B's, so that a lane writes four columns at once.
  auto put = [&](const v16f(&a)[NB], float *to) {
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      // columns of the gate come first, then up's: 32 NB of a wave are 16 NB of each
      const int at = !TWO ? wn * 32 * NB + 32 * j : (j >= NB / 2 ? TB / 2 : 0) + wn * 16 * NB + 32 * (j % (NB / 2));
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<float4 *>(to + (32 * wm + xl) * SLD + at + 2 * r + 4 * h) =
            make_float4(a[j][r], a[j][r + 1], a[j][r + 2], a[j][r + 3]);
    }
  };
  put(acc[0], stage);
#pragma unroll 1
  for (int ps = 0; ps < NB; ++ps) {
    __syncthreads();                             // the band is there, the one before it is read
    float *now = stage + (ps & 1) * BAND * SLD, *next = stage + (~ps & 1) * BAND * SLD;
    if (ps == 0) put(acc[1], next);
    else if (ps == 1 && NB > 2) put(acc[NB - 2], next);
    else if (ps == 2) put(acc[NB - 1], next);
#pragma unroll
    for (int v = 0; v < EACH; ++v) {
      const int row = row_of(ps, v);
      if (row < p.M && col < p.N) {
        const float *x = now + (tid + GP_THREADS * v) / UNITS * SLD + c;
        const int64_t at = (int64_t)row * p.ldc + col;
        if constexpr (EPI == GP_GATED) {
          v4u og, ou, oh;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float g0 = x[2 * e], g1 = x[2 * e + 1], u0 = x[TB / 2 + 2 * e], u1 = x[TB / 2 + 2 * e + 1];
            og[e] = gp_pack(g0, g1);
            ou[e] = gp_pack(u0, u1);
            oh[e] = gp_pack(gp_act<ACT>(g0).a * u0, gp_act<ACT>(g1).a * u1);
          }
          *reinterpret_cast<v4u *>(static_cast<uint16_t *>(p.C[0]) + at) = oh;
          if (p.keep_gate) {
            *reinterpret_cast<v4u *>(p.keep_gate + at) = og;
            *reinterpret_cast<v4u *>(p.keep_up + at) = ou;
          }
        } else if constexpr (EPI == GP_F32 || EPI == GP_PART) {
          float *o = EPI != GP_PART ? static_cast<float *>(p.C[0]) + at
                                   : static_cast<float *>(p.C[0]) +
                                         ((int64_t)blockIdx.y * (TWO ? 2 : 1) + second) * p.M * p.N + (int64_t)row * p.N + col;
          v4f *to = reinterpret_cast<v4f *>(o);
          to[0] = v4f{x[0], x[1], x[2], x[3]};
          to[1] = v4f{x[4], x[5], x[6], x[7]};
        } else if constexpr (EPI == GP_BF16 || EPI == GP_BF16_FAR) {
          v4u o;
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = gp_pack(x[2 * e], x[2 * e + 1]);
          v4u *to = reinterpret_cast<v4u *>(static_cast<uint16_t *>(p.C[0]) + at);
          if constexpr (EPI == GP_BF16_FAR) __builtin_nontemporal_store(o, to);
          else *to = o;
        } else {
          v4u og, ou, oh;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float a[2], b[2], o[2];
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              const float u = gp_float((uint16_t)(ku[0][v][e] >> 16 * w)), d = x[2 * e + w];
              const GpAct f = gp_act<ACT>(gp_float((uint16_t)(kg[0][v][e] >> 16 * w)));
              a[w] = d * u * f.d;
              b[w] = d * f.a;
              o[w] = f.a * u;
            }
            og[e] = gp_pack(a[0], a[1]);
            ou[e] = gp_pack(b[0], b[1]);
            oh[e] = gp_pack(o[0], o[1]);
          }
          kg[0][v] = kg[1][v];
          ku[0][v] = ku[1][v];
          if (ps + 2 < NB) kept(1, ps + 2, v);
          *reinterpret_cast<v4u *>(static_cast<uint16_t *>(p.C[0]) + at) = og;
          *reinterpret_cast<v4u *>(static_cast<uint16_t *>(p.C[1]) + at) = ou;
          *reinterpret_cast<v4u *>(p.hidden + at) = oh;
        }
      }
    }
  }
}

template <bool AK, bool BK, int EPI, int NB, int ACT, bool TWO>
hipError_t gp_tiles(GpParams p, hipStream_t s) {
  constexpr int TB = 64 * NB;
  const int width = TWO ? TB / 2 : TB;
  p.tiles_m = (p.M + TB - 1) / TB;
  p.tiles_n = (p.N + width - 1) / width;
  int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
  for (int i = 0; i < p.others; ++i) {
    GpOther &o = p.other[i];
    o.tiles_m = (o.M + TB - 1) / TB;
    o.tiles_n = (o.N + TB - 1) / TB;
    tiles += (int64_t)o.tiles_m * o.tiles_n;
  }
  const dim3 grid((unsigned)tiles, (unsigned)p.splits), block(GP_THREADS);
  // tiles that have a compute unit of their own may fill its LDS: more slabs on their way (128 x 4096
  // x 14336 forward 126 -> 101 us, 300 x 4096 x 8192 gradients 260 -> 237; two on one take 80 KB each)
  if constexpr (NB == 2 && EPI != GP_BF16_FAR) {   // these have more tiles
    if (tiles * p.splits <= 256) {
      hipLaunchKernelGGL((product_tiles<AK, BK, EPI, NB, ACT, TWO, 9>), grid, block, 0, s, p);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((product_tiles<AK, BK, EPI, NB, ACT, TWO, 5>), grid, block, 0, s, p);
  return hipGetLastError();
}

// Tiles of a product (64 nb on a side) and the parts of k that each is summed in.
struct GpPlan {
  int nb, splits;
};
constexpr int64_t GP_PARTS = (int64_t)256 * 256 * 256 * 4;   // bytes of all parts at most
// By the time of either, in microseconds, from measured kernels (200 to 1500 tokens, 600 to 8192
// wide, both tiles in 1 to 16 parts; within about 15 per cent): a slab of 128-tiles takes 0.62
// where each has a compute unit of its own, 1.05 for two of them on one; of 256-tiles 1.1, and 1.5
// with all compute units busy; starting and writing a tile 4.5 and 9; parts cost a launch for each
// product and their bytes written and read.  Of up to `brief` slabs the outputs are most of a tile's
// time, which two 128-tiles on a compute unit cover for each other (weights' gradients, four: 6 x 4096 x
// 14336 194 us, by 256-tiles 223; 200 x 4096 x 8192 172 and 179; others, two: forward 2000 x 64 x 4096 33.5
// and 35.8, but 4000 x 256 x 8192 132 and 119).
GpPlan gp_plan(const GpParams &p, bool two, int brief) {
  const int64_t w = two ? 2 : 1, slabs = (int64_t)((p.K + GP_KB - 1) / GP_KB) * p.segments;
  GpPlan best{2, 1};
  double least = 1e300;
  for (int nb = 2; nb <= (slabs <= brief ? 2 : 4); nb += 2) {
    const int64_t tb = 64 * nb;
    int64_t tiles = (p.M + tb - 1) / tb * ((w * p.N + tb - 1) / tb), values = (int64_t)p.M * p.N * w;
    for (int i = 0; i < p.others; ++i) {
      tiles += (p.other[i].M + tb - 1) / tb * ((p.other[i].N + tb - 1) / tb);
      values += (int64_t)p.other[i].M * p.other[i].N;
    }
    for (int64_t s = 1; s <= 16 && (s == 1 || slabs / s >= 3); ++s) {
      const int64_t blocks = tiles * s, each = (slabs + s - 1) / s, bytes = 4 * s * values;
      if (s > 1 && (bytes > GP_PARTS || blocks > 1024)) break;
      double t;
      if (nb == 4) t = (double)((blocks + 255) / 256) * (9 + each * (1.1 + 0.4 * std::min(1.0, blocks / 256.0)));
      else t = blocks <= 256 ? 4.5 + 0.62 * each : (double)((blocks + 511) / 512) * (4.5 + 1.05 * each);
      if (s > 1) t += 4 * (1 + p.others) + 0.36e-6 * bytes;
      if (t < least) {
        least = t;
        best = {nb, (int)s};
      }
    }
  }
  return best;
}

// The products, in parts of k and their sum where tiles are few: into `part`.
template <bool AK, bool BK, int EPI, int ACT = SOAP_ACT_SILU>
hipError_t gp_launch(GpParams p, float *part, hipStream_t s) {
  if (p.M <= 0 || p.N <= 0) return hipSuccess;
  constexpr bool TWO = EPI == GP_GATED;
  const GpPlan plan = gp_plan(p, TWO, !AK && !BK ? 4 : 2);
  p.splits = plan.splits;
  if (plan.splits == 1)
    return plan.nb == 4 ? gp_tiles<AK, BK, EPI, 4, ACT, TWO>(p, s) : gp_tiles<AK, BK, EPI, 2, ACT, TWO>(p, s);
  GatedJoin j[3];
  j[0].T = p.M; j[0].N = p.N; j[0].splits = plan.splits; j[0].ldo = p.ldc; j[0].act = ACT;
  j[0].out = static_cast<uint16_t *>(p.C[0]);
  if constexpr (EPI == GP_GATED) {
    j[0].kind = GatedJoin::GATED;
    j[0].keep_gate = p.keep_gate; j[0].keep_up = p.keep_up;
  } else if constexpr (EPI == GP_DGATED) {
    j[0].kind = GatedJoin::DGATED;
    j[0].out2 = static_cast<uint16_t *>(p.C[1]); j[0].hidden = p.hidden; j[0].gate = p.gate; j[0].up = p.up;
  } else if constexpr (EPI == GP_F32) {
    j[0].kind = GatedJoin::F32;
    j[0].out_f32 = static_cast<float *>(p.C[0]);
  }
  j[0].part = part;
  p.C[0] = part;
  for (int i = 0; i < p.others; ++i) {           // each product's parts behind the one before
    GpOther &o = p.other[i];
    j[i + 1] = j[0];
    j[i + 1].T = o.M; j[i + 1].N = o.N; j[i + 1].ldo = o.ldc;
    j[i + 1].out = static_cast<uint16_t *>(o.C); j[i + 1].out_f32 = static_cast<float *>(o.C);
    float *mine = const_cast<float *>(j[i].part) + plan.splits * j[i].T * j[i].N;
    j[i + 1].part = mine;
    o.C = mine;
  }
  hipError_t e = plan.nb == 4 ? gp_tiles<AK, BK, GP_PART, 4, 0, TWO>(p, s) : gp_tiles<AK, BK, GP_PART, 2, 0, TWO>(p, s);
  for (int i = 0; i <= p.others && e == hipSuccess; ++i) e = launch_gated_join(j[i], s);
  return e;
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }
size_t wide(int64_t tokens, int64_t n) { return up256(2 * (size_t)tokens * (size_t)n); }
// Parts of a product of few tokens: 64 columns a workgroup, fewer than 256 workgroups more than
// the columns need.
size_t few_bytes(int64_t tokens, int64_t n, int matrices) {
  return up256(4 * (size_t)std::min(tokens, GATED_FEW) * matrices * 64 * (size_t)((n + 63) / 64 + 256));
}

hipError_t few_fwd(const GatedDesc &d, hipStream_t s) {
  char *w = static_cast<char *>(d.workspace);
  uint16_t *hidden = (uint16_t *)w, *low = (uint16_t *)(w + wide(d.tokens, d.n));
  FewDesc f;
  f.kind = FewDesc::GATE_UP; f.tokens = d.tokens; f.n = d.n; f.k = d.m; f.ldx = d.ldx; f.ldw = d.n;
  f.x[0] = d.x; f.w[0] = d.w_gate; f.w[1] = d.w_up; f.part = (float *)(w + 2 * wide(d.tokens, d.n));
  GatedJoin j;
  j.kind = GatedJoin::GATED; j.act = d.act; j.out = hidden; j.low = low; j.keep_gate = d.gate; j.keep_up = d.up;
  const hipError_t e = launch_product_few(f, j, s);
  if (e != hipSuccess) return e;
  FewDesc g;
  g.kind = FewDesc::HALVES; g.tokens = d.tokens; g.n = d.p; g.k = d.n; g.ldx = d.n; g.ldw = d.p;
  g.x[0] = hidden; g.x[1] = low; g.w[0] = d.w_down; g.part = f.part;
  j = GatedJoin();
  j.out = d.y; j.ldo = d.ldy;
  return launch_product_few(g, j, s);
}

// dG, dU and H, each followed by its lower half, and dX if it is wanted.
hipError_t few_bwd(const GatedDesc &d, uint16_t *const halves[6], float *part, hipStream_t s) {
  FewDesc f;
  f.kind = FewDesc::ROWS; f.tokens = d.tokens; f.n = d.n; f.k = d.p; f.ldx = d.lddy; f.ldw = d.p;
  f.x[0] = d.dy; f.w[0] = d.w_down; f.part = part;
  GatedJoin j;
  j.kind = GatedJoin::DGATED; j.act = d.act; j.gate = d.gate; j.up = d.up;
  j.out = halves[0]; j.low = halves[1]; j.out2 = halves[2]; j.low2 = halves[3]; j.hidden = halves[4]; j.hidden_low = halves[5];
  const hipError_t e = launch_product_few(f, j, s);
  if (e != hipSuccess || !d.dx) return e;
  f = FewDesc();
  f.kind = FewDesc::ROWS_HALVES; f.tokens = d.tokens; f.n = d.m; f.k = d.n; f.ldx = d.n; f.ldw = d.n; f.segments = 2;
  for (int i = 0; i < 4; ++i) f.x[i] = halves[i];
  f.w[0] = d.w_gate; f.w[1] = d.w_up; f.part = part;
  j = GatedJoin();
  j.out = d.dx; j.ldo = d.lddx;
  return launch_product_few(f, j, s);
}

}  // namespace

// H or dG, dU and H, of few tokens with their lower halves, and sums of parts of k.
size_t gated_workspace_bytes(int64_t tokens, int64_t m, int64_t n, int64_t p, bool backward) {
  if (!tokens) return 0;
  const size_t parts = backward ? std::max(few_bytes(tokens, n, 1), few_bytes(tokens, m, 1))
                                : std::max(few_bytes(tokens, n, 2), few_bytes(tokens, p, 1));
  // parts of tiles' products: at most 16, of three slabs each; more tokens never need less
  int64_t tiled = tokens > GATED_FEW ? tokens * (backward ? std::max(m, n) : std::max(2 * n, p)) : 0;
  if (backward && tokens > 5 * GP_KB) tiled = std::max(tiled, n * (2 * m + p));
  tiled = std::min(GP_PARTS, 64 * tiled);
  return (backward ? 3 : 1) * (wide(tokens, n) + wide(std::min(tokens, GATED_FEW), n)) + std::max(parts, up256((size_t)tiled));
}

hipError_t launch_gated_fwd(const GatedDesc &d, hipStream_t s) {
  if (d.tokens <= 0) return hipSuccess;
  if (d.tokens <= GATED_FEW) return few_fwd(d, s);
  uint16_t *hidden = static_cast<uint16_t *>(d.workspace);
  float *part = (float *)(static_cast<char *>(d.workspace) + wide(d.tokens, d.n) + wide(GATED_FEW, d.n));
  GpParams p{};
  p.M = (int)d.tokens; p.N = (int)d.n; p.K = (int)d.m; p.segments = 1;
  p.A[0] = d.x; p.lda = d.ldx; p.B[0] = d.w_gate; p.B[1] = d.w_up; p.ldb = d.n;
  p.C[0] = hidden; p.ldc = d.n; p.keep_gate = d.gate; p.keep_up = d.up;
  hipError_t e = d.act == SOAP_ACT_SILU ? gp_launch<true, false, GP_GATED, SOAP_ACT_SILU>(p, part, s)
                                        : gp_launch<true, false, GP_GATED, SOAP_ACT_GELU>(p, part, s);
  if (e != hipSuccess) return e;
  p = GpParams{};
  p.M = (int)d.tokens; p.N = (int)d.p; p.K = (int)d.n; p.segments = 1;
  p.A[0] = hidden; p.lda = d.n; p.B[0] = d.w_down; p.ldb = d.p;
  p.C[0] = d.y; p.ldc = d.ldy;
  return gp_launch<true, false, GP_BF16>(p, part, s);
}

hipError_t launch_gated_bwd(const GatedDesc &d, hipStream_t s) {
  const bool few = d.tokens <= GATED_FEW;
  const size_t each = wide(d.tokens, d.n), low = few ? each : 0;
  char *w = static_cast<char *>(d.workspace);
  uint16_t *halves[6];
  for (int i = 0; i < 6; ++i) halves[i] = (uint16_t *)(w + (i + 1) / 2 * each + i / 2 * low);
  uint16_t *dg = halves[0], *du = halves[2], *hidden = halves[4];
  float *part = (float *)(w + 3 * (each + low));
  hipError_t e = hipSuccess;
  GpParams p{};
  if (d.tokens > 0 && few) {
    if ((e = few_bwd(d, halves, part, s)) != hipSuccess) return e;
  } else if (d.tokens > 0) {
    p.M = (int)d.tokens; p.N = (int)d.n; p.K = (int)d.p; p.segments = 1;
    p.A[0] = d.dy; p.lda = d.lddy; p.B[0] = d.w_down; p.ldb = d.p;
    p.C[0] = dg; p.C[1] = du; p.hidden = hidden; p.ldc = d.n; p.gate = d.gate; p.up = d.up;
    e = d.act == SOAP_ACT_SILU ? gp_launch<true, true, GP_DGATED, SOAP_ACT_SILU>(p, part, s)
                               : gp_launch<true, true, GP_DGATED, SOAP_ACT_GELU>(p, part, s);
    if (e != hipSuccess) return e;
    if (d.dx) {
      p = GpParams{};
      p.M = (int)d.tokens; p.N = (int)d.m; p.K = (int)d.n; p.segments = 2;
      p.A[0] = dg; p.A[1] = du; p.lda = d.n; p.B[0] = d.w_gate; p.B[1] = d.w_up; p.ldb = d.n;
      p.C[0] = d.dx; p.ldc = d.lddx;
      if ((e = gp_launch<true, true, GP_BF16>(p, part, s)) != hipSuccess) return e;
    }
  }
  // the second segment: lower halves
  p = GpParams{};
  p.K = (int)d.tokens; p.segments = few ? 2 : 1;
  auto grad = [&](int64_t rows, int64_t cols, const uint16_t *a, const uint16_t *a_low, int64_t lda, const uint16_t *b,
                  const uint16_t *b_low, int64_t ldb, void *c) {
    if (!c) return;
    if (!p.M) {
      p.M = (int)rows; p.N = (int)cols; p.lda = lda; p.ldb = ldb; p.ldc = cols;
      p.A[0] = a; p.A[1] = a_low; p.B[0] = b; p.B[1] = b_low; p.C[0] = c;
    } else {
      p.other[p.others++] = GpOther{(int)rows, (int)cols, 0, 0, {a, a_low}, {b, b_low}, c, lda, ldb, cols};
    }
  };
  grad(d.m, d.n, d.x, d.x, d.ldx, dg, halves[1], d.n, d.dw_gate);
  grad(d.m, d.n, d.x, d.x, d.ldx, du, halves[3], d.n, d.dw_up);
  grad(d.n, d.p, hidden, halves[5], d.n, d.dy, d.dy, d.lddy, d.dw_down);
  if (!d.grad_bf16) return gp_launch<false, false, GP_F32>(p, part, s);
  return 2 * d.n * (2 * d.m + d.p) > GP_CACHED ? gp_launch<false, false, GP_BF16_FAR>(p, part, s)
                                               : gp_launch<false, false, GP_BF16>(p, part, s);
}

}  // namespace soap
