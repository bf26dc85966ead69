// Causal linear attention with a decay per head: with lam = exp(log_decay[h]) and
// c = 1 / sqrt(d_k),
//     S_t = lam S_{t-1} + k_t (x) v_t,   y_t = c q_t S_t,
// its gradients and its single step.  All four sums over a sequence (y, dq, dk and
// dv) are one scan with the tensors in other places,
//     out_t = c sum_{s<=t} lam^(t-s) (a_t . b_s) w_s + (the state before the first token),
//     y : a = q,  b = k,  w = v         dq: a = dy, b = v,  w = k
//     dv: a = k,  b = q,  w = dy        dk: a = v,  b = dy, w = q   (from the last token back)
#include <hip/hip_runtime.h>

#include "device_common.hpp"
#include "kernels.hpp"
#include "pair_tiles.hpp"

namespace sata {

namespace {

// exp(g)^e as a float pair.  A single float would do for one factor, but the state is
// multiplied by the same one at every step: its error (2^-25) would grow with the
// number of steps, while the roundings of the products are independent.
struct FloatPair {
  float hi, lo;
};
__device__ __forceinline__ FloatPair decay_power(float g, int e) {
  const double x = e == 0 ? 1.0 : exp((double)g * e);
  const float hi = (float)x;
  return FloatPair{hi, (float)(x - hi)};
}
__device__ __forceinline__ float times(float x, FloatPair p) { return fmaf(x, p.hi, x * p.lo); }

// One workgroup per key/value head, one thread per column of the state, token by token.
template <typename T>
__global__ void __launch_bounds__(kMaxPairDim) decay_scan_kernel(DecayScan s) {
  __shared__ float S[kMaxPairDim][kMaxPairDim];
  __shared__ float xa[kMaxPairDim], xb[kMaxPairDim];
  const int head = blockIdx.x, b = head / s.H, j = threadIdx.x;
  const int len = tokens_of(s.lengths, b, s.n);
  const FloatPair lam = decay_power(s.log_decay[head % s.H], 1);
  if (j < s.dw)
    for (int i = 0; i < s.da; ++i)
      S[i][j] = s.S_in ? s.S_in[(int64_t)head * s.da * s.dw + (s.transposed ? j * s.da + i : i * s.dw + j)] : 0.f;
  for (int u = 0; u < s.n; ++u) {
    const int t = s.reverse ? s.n - 1 - u : u;
    if (t >= len) {
      for (int g = 0; g < s.ga; ++g)
        if (s.out && j < s.dw) ((T*)s.out)[(((int64_t)head * s.ga + g) * s.n + t) * s.dw + j] = from_f32<T>(0.f);
      continue;
    }
    if (!s.reverse && j < s.dw)
      for (int i = 0; i < s.da; ++i) S[i][j] = times(S[i][j], lam);
    for (int g = 0; g < s.gb; ++g) {
      __syncthreads();
      if (j < s.da) xb[j] = to_f32(((const T*)s.b)[(((int64_t)head * s.gb + g) * s.n + t) * s.da + j]);
      __syncthreads();
      if (j < s.dw) {
        const float w = s.update * to_f32(((const T*)s.w)[(((int64_t)head * s.gb + g) * s.n + t) * s.dw + j]);
        for (int i = 0; i < s.da; ++i) S[i][j] = fmaf(xb[i], w, S[i][j]);
      }
    }
    for (int g = 0; g < s.ga; ++g) {
      __syncthreads();
      if (j < s.da) xa[j] = to_f32(((const T*)s.a)[(((int64_t)head * s.ga + g) * s.n + t) * s.da + j]);
      __syncthreads();
      if (s.out && j < s.dw) {
        float o = 0.f;
        for (int i = 0; i < s.da; ++i) o = fmaf(xa[i], S[i][j], o);
        ((T*)s.out)[(((int64_t)head * s.ga + g) * s.n + t) * s.dw + j] = from_f32<T>(o * s.readout);
      }
    }
    if (s.reverse && j < s.dw)
      for (int i = 0; i < s.da; ++i) S[i][j] = times(S[i][j], lam);
  }
  if (s.S_out && j < s.dw)
    for (int i = 0; i < s.da; ++i)
      s.S_out[(int64_t)head * s.da * s.dw + (s.transposed ? j * s.da + i : i * s.dw + j)] = S[i][j];
}

// One workgroup per key/value head, one thread per column of the state.
template <typename T>
__global__ void __launch_bounds__(kMaxPairDim) decay_step_kernel(float* S, const T* q, const T* k, const T* v,
                                                                const float* log_decay, T* y, int H, int G, int dk,
                                                                int dv, float scale) {
  const int64_t head = blockIdx.x;
  const int j = threadIdx.x;
  if (j >= dv) return;
  const FloatPair lam = decay_power(log_decay[head % H], 1);
  float* const s = S + head * dk * dv + j;
  const float w = to_f32(v[head * dv + j]);
  for (int i = 0; i < dk; ++i) s[i * dv] = fmaf(to_f32(k[head * dk + i]), w, times(s[i * dv], lam));
  for (int g = 0; g < G; ++g) {
    float o = 0.f;
    for (int i = 0; i < dk; ++i) o = fmaf(to_f32(q[(head * G + g) * dk + i]), s[i * dv], o);
    y[(head * G + g) * dv + j] = from_f32<T>(o * scale);
  }
}

}  // namespace

hipError_t launch_decay_scan(const DecayScan& s, bool bf16, hipStream_t st) {
  if (bf16) hipLaunchKernelGGL(decay_scan_kernel<bf16_t>, dim3(s.heads), dim3(kMaxPairDim), 0, st, s);
  else hipLaunchKernelGGL(decay_scan_kernel<float>, dim3(s.heads), dim3(kMaxPairDim), 0, st, s);
  return hipGetLastError();
}

hipError_t launch_decay_step(float* S, const void* q, const void* k, const void* v, const float* log_decay, void* y,
                             bool bf16, int heads, int H, int G, int dk, int dv, float scale, hipStream_t st) {
  if (bf16)
    hipLaunchKernelGGL(decay_step_kernel<bf16_t>, dim3(heads), dim3(kMaxPairDim), 0, st, S, (const bf16_t*)q,
                       (const bf16_t*)k, (const bf16_t*)v, log_decay, (bf16_t*)y, H, G, dk, dv, scale);
  else
    hipLaunchKernelGGL(decay_step_kernel<float>, dim3(heads), dim3(kMaxPairDim), 0, st, S, (const float*)q,
                       (const float*)k, (const float*)v, log_decay, (float*)y, H, G, dk, dv, scale);
  return hipGetLastError();
}

}  // namespace sata
