// Powers of a decay exp(log_decay).
#pragma once

#include <hip/hip_runtime.h>

namespace sata {

// exp(g)^e as a float pair.  A single float would do for one factor, but the state is
// multiplied by the same one at every step: its error (2^-25) would grow with the
// number of steps, while the roundings of the products are independent.
struct FloatPair {
  float hi, lo;
};
__device__ __forceinline__ FloatPair decay_power(float g, int e) {
  const double x = exp((double)fmaxf(g, -1e30f) * e);  // (no minus infinity: times 0 it is NaN)
  const float hi = (float)x;
  return FloatPair{hi, (float)(x - hi)};
}
__device__ __forceinline__ float times(float x, FloatPair p) { return fmaf(x, p.hi, x * p.lo); }

}  // namespace sata
