// Exact causal softmax attention: with c = 1 / sqrt(d_k),
//     lse_t = log sum_{s<=t} exp(c q_t.k_s),  p_ts = exp(c q_t.k_s - lse_t),  y_t = sum_{s<=t} p_ts v_s,
// its gradients with the probabilities computed again from lse,
//     dv_s = sum_{t>=s} p_ts dy_t,   e_ts = c p_ts (dy_t.v_s - dy_t.y_t),
//     dq_t = sum_{s<=t} e_ts k_s,    dk_s = sum_{t>=s} e_ts q_t,
// and its single step over a cache.
#include <hip/hip_runtime.h>

#include "device_common.hpp"
#include "kernels.hpp"

namespace sata {

namespace {

__device__ __forceinline__ int tokens_of(const int* lengths, int b, int n) {
  return lengths ? min(max(lengths[b], 0), n) : n;
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int i = 32; i >= 1; i >>= 1) x += __shfl_xor(x, i);
  return x;
}

// A row of up to 128 entries over a wave: entries lane and lane + 64.
template <typename T>
__device__ __forceinline__ float2 row_of(const T* p, int d) {
  const int l = threadIdx.x;
  return float2{l < d ? to_f32(p[l]) : 0.f, l + 64 < d ? to_f32(p[l + 64]) : 0.f};
}
template <typename T>
__device__ __forceinline__ void put_row(T* p, int d, float2 x) {
  const int l = threadIdx.x;
  if (l < d) p[l] = from_f32<T>(x.x);
  if (l + 64 < d) p[l + 64] = from_f32<T>(x.y);
}
__device__ __forceinline__ float dot(float2 a, float2 b) { return wave_sum(fmaf(a.x, b.x, a.y * b.y)); }

// One wave per query: keys one after the other, running maximum and sum.
template <typename T>
__device__ __forceinline__ float attend(const T* q, const T* k, const T* v, int keys, int dk, int dv, float c, float2& y) {
  const float2 x = row_of(q, dk);
  float m = -INFINITY, l = 0.f;
  y = float2{0.f, 0.f};
  for (int s = 0; s < keys; ++s) {
    const float z = c * dot(x, row_of(k + (int64_t)s * dk, dk));
    const float top = fmaxf(m, z), base = top == -INFINITY ? 0.f : top;
    const float keep = expf(m - base), p = expf(z - base);
    const float2 w = row_of(v + (int64_t)s * dv, dv);
    l = l * keep + p;
    y.x = y.x * keep + p * w.x;
    y.y = y.y * keep + p * w.y;
    m = top;
  }
  const float r = keys > 0 ? 1.f / l : 0.f;
  y.x *= r, y.y *= r;
  return keys > 0 ? logf(l) + m : -INFINITY;
}

template <typename T>
__global__ void __launch_bounds__(64) softmax_prefill_kernel(SoftmaxArgs a) {
  const int t = blockIdx.x;
  const int64_t qh = blockIdx.y, kvh = qh / a.G;
  const int len = tokens_of(a.lengths, (int)(kvh / a.H), a.n);
  float2 y;
  const float lse = attend((const T*)a.q + (qh * a.n + t) * a.dk_, (const T*)a.k + kvh * a.n * a.dk_,
                           (const T*)a.v + kvh * a.n * a.dv_, t < len ? t + 1 : 0, a.dk_, a.dv_, a.scale, y);
  put_row((T*)a.y + (qh * a.n + t) * a.dv_, a.dv_, y);
  if (a.lse && threadIdx.x == 0) a.lse[qh * a.n + t] = lse;
}

template <typename T>
__global__ void __launch_bounds__(64) softmax_rows_kernel(SoftmaxGradArgs a) {
  const int t = blockIdx.x;
  const int64_t qh = blockIdx.y, kvh = qh / a.G;
  const int len = tokens_of(a.lengths, (int)(kvh / a.H), a.n);
  float2 o = {0.f, 0.f};
  if (t < len) {
    const float2 x = row_of((const T*)a.q + (qh * a.n + t) * a.dk_, a.dk_);
    const float2 d = row_of((const T*)a.dy + (qh * a.n + t) * a.dv_, a.dv_);
    const float delta = dot(d, row_of((const T*)a.y + (qh * a.n + t) * a.dv_, a.dv_));
    const float lse = a.lse[qh * a.n + t];
    if (threadIdx.x == 0) a.delta[qh * a.n + t] = delta;
    for (int s = 0; s <= t; ++s) {
      const float2 k = row_of((const T*)a.k + (kvh * a.n + s) * a.dk_, a.dk_);
      const float p = expf(a.scale * dot(x, k) - lse);
      const float e = a.scale * p * (dot(d, row_of((const T*)a.v + (kvh * a.n + s) * a.dv_, a.dv_)) - delta);
      o.x = fmaf(e, k.x, o.x);
      o.y = fmaf(e, k.y, o.y);
    }
  }
  put_row((T*)a.dq + (qh * a.n + t) * a.dk_, a.dk_, o);
}

template <typename T>
__global__ void __launch_bounds__(64) softmax_cols_kernel(SoftmaxGradArgs a) {
  const int s = blockIdx.x;
  const int64_t kvh = blockIdx.y;
  const int len = tokens_of(a.lengths, (int)(kvh / a.H), a.n);
  float2 gk = {0.f, 0.f}, gv = {0.f, 0.f};
  if (s < len) {
    const float2 k = row_of((const T*)a.k + (kvh * a.n + s) * a.dk_, a.dk_);
    const float2 v = row_of((const T*)a.v + (kvh * a.n + s) * a.dv_, a.dv_);
    for (int64_t qh = kvh * a.G; qh < (kvh + 1) * a.G; ++qh)
      for (int t = s; t < len; ++t) {
        const float2 x = row_of((const T*)a.q + (qh * a.n + t) * a.dk_, a.dk_);
        const float2 d = row_of((const T*)a.dy + (qh * a.n + t) * a.dv_, a.dv_);
        const float p = expf(a.scale * dot(x, k) - a.lse[qh * a.n + t]);
        const float e = a.scale * p * (dot(d, v) - a.delta[qh * a.n + t]);
        gk.x = fmaf(e, x.x, gk.x), gk.y = fmaf(e, x.y, gk.y);
        gv.x = fmaf(p, d.x, gv.x), gv.y = fmaf(p, d.y, gv.y);
      }
  }
  put_row((T*)a.dk + (kvh * a.n + s) * a.dk_, a.dk_, gk);
  put_row((T*)a.dv + (kvh * a.n + s) * a.dv_, a.dv_, gv);
}

// One wave per query head; the first member of a group writes the cache.
template <typename T>
__global__ void __launch_bounds__(64) softmax_step_kernel(SoftmaxStepArgs a) {
  const int64_t kvh = blockIdx.x;
  const int at = a.lengths[kvh / a.H];
  const bool on = at >= 0 && at < a.capacity;
  T* const K = (T*)a.K + kvh * a.capacity * a.dk_;
  T* const V = (T*)a.V + kvh * a.capacity * a.dv_;
  if (on) {
    put_row(K + (int64_t)at * a.dk_, a.dk_, row_of((const T*)a.k + kvh * a.dk_, a.dk_));
    put_row(V + (int64_t)at * a.dv_, a.dv_, row_of((const T*)a.v + kvh * a.dv_, a.dv_));
  }
  for (int64_t qh = kvh * a.G; qh < (kvh + 1) * a.G; ++qh) {
    float2 y;
    attend((const T*)a.q + qh * a.dk_, K, V, on ? at + 1 : 0, a.dk_, a.dv_, a.scale, y);
    put_row((T*)a.y + qh * a.dv_, a.dv_, y);
  }
}

}  // namespace

hipError_t launch_softmax_prefill(const SoftmaxArgs& a, bool bf16, hipStream_t s) {
  const dim3 grid(a.n, a.heads * a.G);
  if (bf16) hipLaunchKernelGGL(softmax_prefill_kernel<bf16_t>, grid, dim3(64), 0, s, a);
  else hipLaunchKernelGGL(softmax_prefill_kernel<float>, grid, dim3(64), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_softmax_backward(const SoftmaxGradArgs& a, bool bf16, hipStream_t s) {
  if (bf16) hipLaunchKernelGGL(softmax_rows_kernel<bf16_t>, dim3(a.n, a.heads * a.G), dim3(64), 0, s, a);
  else hipLaunchKernelGGL(softmax_rows_kernel<float>, dim3(a.n, a.heads * a.G), dim3(64), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (bf16) hipLaunchKernelGGL(softmax_cols_kernel<bf16_t>, dim3(a.n, a.heads), dim3(64), 0, s, a);
  else hipLaunchKernelGGL(softmax_cols_kernel<float>, dim3(a.n, a.heads), dim3(64), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_softmax_step(const SoftmaxStepArgs& a, bool bf16, hipStream_t s) {
  if (bf16) hipLaunchKernelGGL(softmax_step_kernel<bf16_t>, dim3(a.heads), dim3(64), 0, s, a);
  else hipLaunchKernelGGL(softmax_step_kernel<float>, dim3(a.heads), dim3(64), 0, s, a);
  return hipGetLastError();
}

}  // namespace sata
