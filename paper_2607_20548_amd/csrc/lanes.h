// Reductions over aligned groups of 8, 16, 32 or 64 lanes of a wave, in registers
// (DPP moves up to 16 lanes, row and half swaps past them): a fixed tree, every lane
// gets the result, all of a group's lanes the same bits.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace soap {

// The value of another lane of the same 16: CTRL 0xB1 lane ^ 1, 0x4E lane ^ 2, 0x141
// 7 - lane of its 8, 0x140 15 - lane of its 16.
template <int CTRL>
__device__ __forceinline__ uint32_t lane_dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}

template <int LANES, typename T, typename F>
__device__ __forceinline__ T lane_reduce(T v, F op) {
  static_assert(LANES >= 8 && LANES <= 64 && (LANES & (LANES - 1)) == 0, "8 to 64 lanes");
  static_assert(sizeof(T) == 4, "32-bit values");
  auto cast = [](uint32_t u) { return __builtin_bit_cast(T, u); };
  auto bits = [](T t) { return __builtin_bit_cast(uint32_t, t); };
  v = op(v, cast(lane_dpp<0xB1>(bits(v))));
  v = op(v, cast(lane_dpp<0x4E>(bits(v))));
  v = op(v, cast(lane_dpp<0x141>(bits(v))));
  if constexpr (LANES >= 16) v = op(v, cast(lane_dpp<0x140>(bits(v))));
  if constexpr (LANES >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(bits(v), bits(v), false, false);
    v = op(cast(r[0]), cast(r[1]));
  }
  if constexpr (LANES >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(bits(v), bits(v), false, false);
    v = op(cast(r[0]), cast(r[1]));
  }
  return v;
}

template <int LANES>
__device__ __forceinline__ float lane_sum(float v) {
  return lane_reduce<LANES>(v, [](float a, float b) { return a + b; });
}
template <int LANES>
__device__ __forceinline__ uint32_t lane_max(uint32_t v) {
  return lane_reduce<LANES>(v, [](uint32_t a, uint32_t b) { return max(a, b); });
}

}  // namespace soap
