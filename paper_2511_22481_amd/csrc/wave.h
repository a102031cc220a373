// A wave's 64 numbers joined by an operation that is its own order's (maximum, minimum, or), without LDS.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace omniattn {

template <typename F>
__device__ __forceinline__ uint32_t wave_join(uint32_t x, F f) {
#define OMNIATTN_JOIN(ctrl) x = f(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, 0xf, 0xf, true))
  OMNIATTN_JOIN(0xb1);   // the other of two
  OMNIATTN_JOIN(0x4e);   // the other two of four
  OMNIATTN_JOIN(0x141);  // eight, mirrored
  OMNIATTN_JOIN(0x140);  // sixteen, mirrored
#undef OMNIATTN_JOIN
  const auto y = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = f(y[0], y[1]);
  const auto z = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)f(z[0], z[1]));
}

}  // namespace omniattn
