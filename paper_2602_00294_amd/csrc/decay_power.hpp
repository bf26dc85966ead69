// Powers of a decay exp(log_decay).
#pragma once

#include <hip/hip_runtime.h>

namespace sata {

// log_decay in double (no minus infinity: times 0 it would be NaN).
__device__ __forceinline__ double decay_rate(float log_decay) { return (double)fmaxf(log_decay, -1e30f); }

// A factor as a float pair.  A single float would do once, but a state is multiplied by the
// same factor at every step: its error (2^-25) would grow with the number of steps, while
// the roundings of the products are independent.
struct FloatPair {
  float hi, lo;
};
__device__ __forceinline__ FloatPair float_pair(double x) {
  const float hi = (float)x;
  return FloatPair{hi, (float)(x - hi)};
}
__device__ __forceinline__ float times(float x, FloatPair p) { return fmaf(x, p.hi, x * p.lo); }

}  // namespace sata
