// Values exchanged between a wave's lanes.
#pragma once

#include <hip/hip_runtime.h>

namespace sru {

// x of lane l ^ O, without LDS for O up to 15; both lanes take part.
template <int O>
__device__ __forceinline__ unsigned lane_xor(unsigned x) {
  constexpr int dpp = O == 1 ? 0xB1 : O == 2 ? 0x4E : O == 3 ? 0x1B  // within four lanes
                      : O == 7 ? 0x141 : O == 15 ? 0x140              // mirrored in 8, 16
                      : O == 8 ? 0x128 : 0;                           // rotated by 8 in 16
  if constexpr (O == 4)
    return lane_xor<3>(lane_xor<7>(x));
  else if constexpr (dpp != 0)
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, dpp, 0xf, 0xf, true);
  else
    return (unsigned)__shfl_xor((int)x, O);
}
// Of LANES consecutive lanes, the same in each: pairs, fours, then mirrored eights
// and sixteens.
template <int LANES, typename F>
__device__ __forceinline__ float lanes_reduce(float x, F f) {
  const auto with = [&](unsigned o) { x = f(x, __uint_as_float(o)); };
  if constexpr (LANES > 1) with(lane_xor<1>(__float_as_uint(x)));
  if constexpr (LANES > 2) with(lane_xor<2>(__float_as_uint(x)));
  if constexpr (LANES > 4) with(lane_xor<7>(__float_as_uint(x)));
  if constexpr (LANES > 8) with(lane_xor<15>(__float_as_uint(x)));
  if constexpr (LANES > 16) with(lane_xor<16>(__float_as_uint(x)));
  if constexpr (LANES > 32) with(lane_xor<32>(__float_as_uint(x)));
  return x;
}
template <int LANES>
__device__ __forceinline__ float lanes_max(float x) {
  return lanes_reduce<LANES>(x, [](float a, float b) { return fmaxf(a, b); });
}
// Not contracted with a product that makes x: a lane's own would enter unrounded,
// its neighbour's rounded, and the lanes' sums would differ.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
  return lanes_reduce<LANES>(x, [](float a, float b) {
#pragma clang fp contract(off)
    return a + b;
  });
}

}  // namespace sru
