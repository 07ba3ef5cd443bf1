// Reductions over the 64 lanes of a wave.
#pragma once

#include "ef_device.hpp"

namespace ef {

// Reductions over the wave's lanes, in DPP moves and lane swaps.
template <class T, class F>
__device__ __forceinline__ T wave_reduce(T x, F f) {
  static_assert(sizeof(T) == 4, "a lane register");
  auto bits = [](T v) { return __builtin_bit_cast(float, v); };
  auto val = [](float v) { return __builtin_bit_cast(T, v); };
  x = f(x, val(dpp_mov<kDppQuadXor1>(bits(x))));
  x = f(x, val(dpp_mov<kDppQuadXor2>(bits(x))));
  x = f(x, val(dpp_mov<kDppHalfMirror>(bits(x))));
  x = f(x, val(dpp_mov<kDppRowRor8>(bits(x))));
  float a, b;
  lane_pair<16>(bits(x), a, b);
  x = f(val(a), val(b));
  lane_pair<32>(bits(x), a, b);
  return f(val(a), val(b));
}
__device__ __forceinline__ float wave_max(float x) {
  return wave_reduce(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  return wave_reduce(x, [](uint32_t a, uint32_t b) { return max(a, b); });
}
__device__ __forceinline__ uint32_t wave_min(uint32_t x) { return ~wave_max(~x); }
__device__ __forceinline__ int wave_min(int x) {
  return wave_reduce(x, [](int a, int b) { return min(a, b); });
}
__device__ __forceinline__ float wave_sum(float x) {
  return wave_reduce(x, [](float a, float b) { return a + b; });
}

}  // namespace ef
