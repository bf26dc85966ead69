// Powers of a decay exp(log_decay).
#pragma once

#include <hip/hip_runtime.h>

namespace sata {

// log_decay in double (no minus infinity: times 0 it would be NaN; NaN stays what it is).
__device__ __forceinline__ double decay_rate(float log_decay) { return log_decay < -1e30f ? -1e30 : (double)log_decay; }
// lam^e.  lam^0 is 1, whatever lam is: a token's share of its own output knows no decay.
__device__ __forceinline__ double decay_power(double rate, int e) { return e == 0 ? 1.0 : exp(rate * e); }

// A token's own log decay in double.  Below -200 a state's entries are zero afterwards, as float32 has none so
// small, and sums of such numbers keep their differences (minus infinity does not); NaN stays.
__device__ __forceinline__ double delta_rate(float g) { return g < -200.f ? -200.0 : (double)g; }

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
