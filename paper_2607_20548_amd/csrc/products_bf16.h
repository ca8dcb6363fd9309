// What the bfloat16 products of the gated feed-forward block share: loads that write LDS
// themselves, operands as bounded buffers, fragments in either orientation, activations.
#pragma once

#include "soap.h"

#include "internal.h"

namespace soap {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) v4s lds_v4s;
typedef int v4i __attribute__((ext_vector_type(4)));

constexpr int GP_THREADS = 256;                  // four waves
constexpr int GP_RSRC = 0x00020000;              // raw 32-bit data

__device__ __forceinline__ uint16_t gp_round(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ float gp_float(uint16_t h) { return __uint_as_float((uint32_t)h << 16); }

// The activation, and its derivative, to their own size: within x^2 2^-24 (the exponential's argument,
// rounded twice) and 1e-6 of it, less than the 2^-16 of the two bfloat16 that few tokens keep as far
// as the results are normal numbers.  The hardware's exponential and reciprocal are within an fp32
// step each.  The normal distribution's function is exp(-x^2 / 2) t P(t) below 0, t = 1 / (1 + 0.3 |x|),
// P of degree 7 fitted to the least largest relative error there, 1.5e-7 for |x| to 14; the
// exponential is the derivative's too (8192 x 2048 x 8192 forward 722 us, by erff 776; by Hastings' five
// terms, whose relative error is 5e-4 at -4 and past bfloat16's rounding from -5.3 on, 723).
struct GpAct {
  float a, d;
};
template <int ACT>
__device__ __forceinline__ GpAct gp_act(float x) {
  GpAct r;
  if constexpr (ACT == SOAP_ACT_SILU) {
    const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * -1.44269504088896340736f));
    r.a = x * s;
    r.d = fmaf(r.a, 1.f - s, s);
  } else {
    const float e = __builtin_amdgcn_exp2f(x * x * -0.72134752044448170368f);
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(x), 0.3f, 1.f));
    float p = fmaf(t, 0.035674773156642914f, -0.1572030782699585f);
    p = fmaf(t, fmaf(t, fmaf(t, p, 0.20635348558425903f), -0.053683631122112274f), 0.1285616159439087f);
    p = fmaf(t, fmaf(t, fmaf(t, p, 0.09991349279880524f), 0.12075395882129669f), 0.11962930113077164f);
    const float q = t * p * e, c = x < 0.f ? q : 1.f - q;
    r.a = x * c;
    r.d = fmaf(x * 0.39894228040143267794f, e, c);
  }
  return r;
}
__device__ __forceinline__ uint32_t gp_pack(float a, float b) { return gp_round(a) | (uint32_t)gp_round(b) << 16; }

// What one operand's blocks of a slab are loaded from: the tile's first row of its matrix, or of
// the slab's k, and the bytes from there to the matrix' end.
struct GpSource {
  const char *base;
  int64_t left, step;          // step: to the next slab
  // kc: rows of x, contiguous along k; otherwise rows of k.  slab: its k.
  __device__ __forceinline__ void start(const uint16_t *q, bool kc, int x0, int X, int K, int64_t ld2, int slab) {
    base = (const char *)q + (kc ? x0 * ld2 : 2 * (int64_t)x0);
    left = kc ? (X - x0 - 1) * ld2 + 2 * (int64_t)K : (K - 1) * ld2 + 2 * (int64_t)(X - x0);
    step = kc ? 2 * slab : slab * ld2;
  }
  __device__ __forceinline__ void next(int64_t slabs = 1) {
    base += slabs * step;
    left -= slabs * step;
  }
  // Offsets stay below 2^31 (rows of a tile are at most 256, of 2^22 bytes).
  __device__ __forceinline__ v4i buffer() const {
    const int hi = (int)(left >> 32);
    const uint32_t lo = (uint32_t)left;
    const uint32_t n = hi < 0 ? 0u : hi > 0 || lo > 0x7fffffffu ? 0x7fffffffu : lo;
    const uint64_t a = reinterpret_cast<uint64_t>(base);
    v4i r = {(int)(uint32_t)a, (int)(uint32_t)(a >> 32) & 0xffff, (int)n, GP_RSRC};
    // five wait states between a vector instruction that may have written it and the loads
    asm volatile("s_nop 4" : "+s"(r));
    return r;
  }
};
constexpr uint32_t GP_OUT = 0x80000000u;         // in an offset: past every buffer's end

// 16 bytes a lane from `offset` of a buffer to LDS at `lds` + 16 lane.  Written out because the
// compiler holds every transposing read until all such loads have arrived; the kernel waits for
// them itself, before the barrier in front of their slab's first read.  They write no register.
// FAR: past the caches.
template <bool FAR = false>
__device__ __forceinline__ void gp_load(const v4i &buffer, uint32_t lds, uint32_t offset) {
  if constexpr (FAR)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(lds), "v"(offset), "s"(buffer)
                 : "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(buffer)
                 : "m0");
}

// The eight k from 8 h on, h = lane / 32, of row lane % 32 of two half blocks: the transposing
// reads give a lane four k of its own x, `rows` bytes apart, from `at` (which its k and x choose).
__device__ __forceinline__ v8bf gp_read_transposed(const uint8_t *at, int rows) {
  const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)at);
  const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(at + 4 * rows));
  return __builtin_bit_cast(v8bf, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

}  // namespace
}  // namespace soap
