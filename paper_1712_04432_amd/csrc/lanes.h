// Exchanges between the lanes of a wave.
#pragma once

#include "common.h"

namespace imbd {

// The value of the lane that a group's reduction pairs with at distance o: inside 16 lanes by the cross-lane forms
// of the vector instructions (at 4 and 8 the mirrored lane, which holds the same as its neighbours by then).
template <int o>
__device__ __forceinline__ int partner(int v) {
  if constexpr (o == 1) return __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, false);        // quad: 1 0 3 2
  else if constexpr (o == 2) return __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, false);   // quad: 2 3 0 1
  else if constexpr (o == 4) return __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, false);  // half rows mirrored
  else if constexpr (o == 8) return __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, false);  // rows mirrored
  else return __shfl_xor(v, o, 64);
}
template <int o>
__device__ __forceinline__ float partner(float v) {
  return __builtin_bit_cast(float, partner<o>(__builtin_bit_cast(int, v)));
}
template <int o>
__device__ __forceinline__ uint64_t partner(uint64_t v) {
  return ((uint64_t)(uint32_t)partner<o>((int)(v >> 32)) << 32) | (uint32_t)partner<o>((int)v);
}

// f over all lanes of the wave, the same value (and bits) in each.
template <typename V, typename F>
__device__ __forceinline__ V wave_all(V v, F f) {
  v = f(v, partner<1>(v));
  v = f(v, partner<2>(v));
  v = f(v, partner<4>(v));
  v = f(v, partner<8>(v));
  v = f(v, partner<16>(v));
  return f(v, partner<32>(v));
}
__device__ __forceinline__ float wave_sum(float v) {
  asm("" : "+v"(v));  // (rounded: a product fused with the first addition would be exact in its own lane only)
  return wave_all(v, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float wave_max(float v) {  // (a NaN is left out)
  return wave_all(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_maximum(float v) {  // (a NaN stays one)
  return wave_all(v, [](float a, float b) { return __builtin_elementwise_maximum(a, b); });
}
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
  return wave_all(v, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
}

}  // namespace imbd
