// Sums and maxima over consecutive lanes of a wave, on the vector units (DPP and
// lane swaps) and without the trip through LDS of a general shuffle, which six
// dependent steps make felt: layer norm of 16384 x 2048 bf16, both ways, 77.5 us
// with shuffles and 74.3 so.
#pragma once

#include "device.h"

namespace ffmlp {

// op(v of this lane, v of the lane whose number differs in bit D).  Steps of 4 and
// 8 mirror their lanes, which is the same where lanes that differ in lower bits
// only hold the same v.
template <int D, typename F>
__device__ __forceinline__ float lanes_step(float v, F&& op) {
  const uint32_t x = __float_as_uint(v);
  if constexpr (D >= 16) {
    const auto s = D == 16 ? __builtin_amdgcn_permlane16_swap(x, x, false, false) : __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return op(__uint_as_float(s[0]), __uint_as_float(s[1]));
  } else {
    // lanes 1 0 3 2 and 2 3 0 1 of four; eight mirrored; sixteen mirrored
    constexpr int ctrl = D == 1 ? 0xb1 : D == 2 ? 0x4e : D == 4 ? 0x141 : 0x140;
    return op(v, __uint_as_float(__builtin_amdgcn_mov_dpp((int)x, ctrl, 0xf, 0xf, true)));
  }
}
// Over groups of LANES lanes (a power of two), every lane with the result.  With
// FROM over the lanes that differ in bits FROM .. LANES / 2 only: 16 and 32, which
// take exactly those lanes, or 1.
template <int LANES, int FROM = 1, typename F>
__device__ __forceinline__ float lanes_all(float v, F&& op) {
  if constexpr (FROM < LANES) return lanes_all<LANES, 2 * FROM>(lanes_step<FROM>(v, op), op);
  else return v;
}
template <int LANES, int FROM = 1>
__device__ __forceinline__ float lanes_sum(float v) {
  return lanes_all<LANES, FROM>(v, [](float a, float b) { return a + b; });
}
template <int LANES, int FROM = 1>
__device__ __forceinline__ float lanes_max(float v) {
  return lanes_all<LANES, FROM>(v, [](float a, float b) { return __builtin_fmaxf(a, b); });
}

}  // namespace ffmlp
