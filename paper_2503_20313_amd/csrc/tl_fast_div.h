// Division by a number the host knows.
#pragma once
#include <hip/hip_runtime.h>

namespace tl {

// n / d for 0 <= n < 2^31 as a multiplication by a 32-bit reciprocal (the round-up method of Granlund and Montgomery,
// "Division by Invariant Integers using Multiplication", 1994: m = floor(2^32 (2^l - d) / d) + 1
// with l = ceil(log2 d), n / d = (mulhi(m, n) + n) >> l).
struct FastDiv {
  unsigned mul, shift;
  __device__ __forceinline__ unsigned div(unsigned n) const { return (__umulhi(mul, n) + n) >> shift; }
};
inline FastDiv make_fast_div(unsigned d) {
  FastDiv f;
  f.shift = 0;
  while (f.shift < 31 && (1u << f.shift) < d) f.shift++;
  f.mul = (unsigned)((((1ull << f.shift) - d) << 32) / d + 1);
  return f;
}

}  // namespace tl
