// Floats as whole numbers of the same order, for choices by value.
#pragma once

#include "common.h"

namespace imbd {

// Whole number of the same order as v; NaN the largest, 0 is below every value.
__device__ __forceinline__ uint32_t order_key(float v) {
  if (v != v) return 0xffffffffu;
  const uint32_t u = __builtin_bit_cast(uint32_t, v + 0.0f);  // (-0 becomes +0: they tie)
  return (u >> 31) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  if (k == 0xffffffffu) return __builtin_nanf("");
  return __builtin_bit_cast(float, (k >> 31) ? (k & 0x7fffffffu) : ~k);
}
constexpr uint32_t KEY_MINUS_INF = 0x007fffffu;  // order_key(-inf)

}  // namespace imbd
