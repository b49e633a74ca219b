// The angle of a pair at a position, pos * inv_freq radians, without the whole turns in it: the same on the host (where it is tested) and on the device.
//
// A position has 31 bits and a frequency 24; formed in fp64, pos * (f / 2 pi) is off by 4.5e-7 radians at pos = 2^31, f = 1, and by as much more as f is
// larger.  But positions are whole numbers, so whole turns of f / 2 pi itself are whole turns at every position: what is left of it is held
// in 2^-64 of a turn, and a product that wraps around drops the turns by itself.  f / 2 pi comes as q + e, from 1 / 2 pi in two pieces and what the products
// leave behind, right to 2^-104 of itself; so while |f| is 2^40 at most, the number is off by 1 (two roundings to whole numbers), a position's part of a turn
// by 2^-33 (7e-10 radians), and what counts is its rounding to fp32.
#pragma once
#include <stdint.h>
#ifdef __CUDACC__
#define MST_ANGLE_HD __host__ __device__ __forceinline__
#else
#include <cmath>
#define MST_ANGLE_HD inline
#endif

namespace mst_rot {

// what a position adds, in 2^-64 of a turn; any number for a frequency that is not finite
MST_ANGLE_HD uint64_t step_of(float inv_freq) {
  constexpr double HI = 0x1.45f306dc9c883p-3, LO = -0x1.6b01ec5417056p-57;     // 1 / 2 pi to 2^-110
  constexpr double ONE = 18446744073709551616.0;
  const double f = inv_freq;
#ifdef __CUDA_ARCH__
  const double q = __dmul_rn(f, HI), e = __fma_rn(f, LO, __fma_rn(f, HI, -q));
  return (uint64_t)__double2ll_rn((q - rint(q)) * ONE) + (uint64_t)__double2ll_rn((e - rint(e)) * ONE);
#else
  const double q = f * HI, e = std::fma(f, LO, std::fma(f, HI, -q));
  return (uint64_t)llrint((q - rint(q)) * ONE) + (uint64_t)llrint((e - rint(e)) * ONE);
#endif
}
// of a position: half turns between -1 and 1
MST_ANGLE_HD float half_turns(uint64_t step, int pos) { return (float)(int64_t)(step * (uint64_t)(int64_t)pos) * 0x1p-63f; }

}  // namespace mst_rot
