// Prefix sums over a wave, by lane moves.
#pragma once

#include "common.hpp"

namespace baton {

// One step of a wave's prefix sum: x plus the value DPP moves here (0 from outside).
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t dpp_add(uint64_t x) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, ROWS, 0xF, false);
  return x + ((uint64_t)hi << 32 | lo);
}
// Inclusive prefix sum over the wave: within rows of 16 lanes, then across them.
__device__ __forceinline__ uint64_t wave_scan(uint64_t x) {
  x = dpp_add<0x111, 0xF>(x);   // row_shr 1, 2, 4, 8
  x = dpp_add<0x112, 0xF>(x);
  x = dpp_add<0x114, 0xF>(x);
  x = dpp_add<0x118, 0xF>(x);
  x = dpp_add<0x142, 0xA>(x);   // lane 15 of each row into the next (rows 1 and 3)
  x = dpp_add<0x143, 0xC>(x);   // lane 31 into the upper half
  return x;
}

}  // namespace baton
