// Lane-level pieces of the online softmax over 32x32 score tiles, shared by the attention kernels.  gfx950 only.
#pragma once
#include "tl_device.h"

namespace tl {

// The two values a query column has in lanes l and l+32, in every lane (one VALU lane-half swap, no LDS round trip).
__device__ __forceinline__ void both_halves(float v, float& lo, float& hi) {
  const unsigned b = __builtin_bit_cast(unsigned, v);
  auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  lo = __builtin_bit_cast(float, (unsigned)r[0]);
  hi = __builtin_bit_cast(float, (unsigned)r[1]);
}
// max(a, b) of two raw matrix-instruction results.  Written as a median with +inf, which the compiler turns into one
// v_max_f32 on the raw registers; fmaxf() on them would first canonicalise each operand with an instruction of its own.
__device__ __forceinline__ float raw_max(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, __builtin_inff()); }

// max(m, a, b) in one instruction on raw matrix-instruction results (finite or -inf).  The compiler does not look into it
// and keeps no distance from the matrix instruction that writes a or b: only where at least two later matrix instructions
// stand in between and cover that one's latency; raw_max() elsewhere.
__device__ __forceinline__ float raw_max3(float m, float a, float b) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(m), "v"(a), "v"(b));
  return r;
}

__device__ __forceinline__ float halves_max(float v) {
  float lo, hi;
  both_halves(v, lo, hi);
  return __builtin_fmaxf(lo, hi);
}

}  // namespace tl
