// One token of linear attention with a decay: S = lam S + k (x) v, y = c q S.
//
// Bound: the state is read and written once, 8 d_k d_v bytes a head.  A workgroup holds a
// head's whole state in registers, a thread R rows of V columns, all loaded at once; the G
// query heads of the group are read out of the registers, four at a time, and
// their rows' sums joined in LDS.  The state is streamed (nontemporal): a model's states are more than
// the caches hold.  2048 heads of d = 128 in groups of four, 268 MB: 58.9 us (4.66 TB/s; a copy
// of 4 GB 4.9); 75.9 with plain loads and stores, 69 with one of the two; 60.2 against
// 56.6 where the states of the last call still lie in the 256 MB cache.  512 and 128
// threads 89 and 82 us.
#include <hip/hip_runtime.h>

#include "decay_power.hpp"
#include "device_common.hpp"
#include "kernels.hpp"

namespace sata {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kStepThreads = 256;
constexpr int kMembers = 4;  // query heads read out at a time

// V: columns of a thread (4: whole 16-byte vectors; 1); R: rows of a thread at most.
template <typename T, int V, int R>
__global__ void __launch_bounds__(kStepThreads) decay_step_kernel(float* __restrict__ S_, const T* __restrict__ q_,
                                                                  const T* __restrict__ k_, const T* __restrict__ v_,
                                                                  const float* __restrict__ log_decay,
                                                                  T* __restrict__ y_, int H, int G, int dk, int dv,
                                                                  float scale) {
  __shared__ float qs[kMembers][kMaxPairDim];
  __shared__ float sums[kMembers * kStepThreads * V];  // [member][row group][column]
  const int64_t head = blockIdx.x;
  const int tid = threadIdx.x, cols = dv / V, groups = kStepThreads / cols;
  const int rg = tid / cols, c0 = (tid - rg * cols) * V;
  const bool on = rg < groups;
  float* const S = S_ + head * dk * dv + c0;
  float s[R][V], w[V];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int row = rg + i * groups;
#pragma unroll
    for (int x = 0; x < V; ++x) s[i][x] = 0.f;
    if (on && row < dk) {
      if constexpr (V == 4) {
        const f32x4 f = __builtin_nontemporal_load((const f32x4*)(S + row * dv));
#pragma unroll
        for (int x = 0; x < 4; ++x) s[i][x] = f[x];
      } else {
        s[i][0] = S[row * dv];
      }
    }
  }
#pragma unroll
  for (int x = 0; x < V; ++x) w[x] = on ? to_f32(v_[head * dv + c0 + x]) : 0.f;
  const FloatPair lam = float_pair(exp(decay_rate(log_decay[head % H])));
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int row = rg + i * groups;
    if (on && row < dk) {
      const float k = to_f32(k_[head * dk + row]);
#pragma unroll
      for (int x = 0; x < V; ++x) s[i][x] = fmaf(k, w[x], times(s[i][x], lam));
      if constexpr (V == 4) __builtin_nontemporal_store(f32x4{s[i][0], s[i][1], s[i][2], s[i][3]}, (f32x4*)(S + row * dv));
      else S[row * dv] = s[i][0];
    }
  }
  for (int g0 = 0; g0 < G; g0 += kMembers) {
    const int members = min(kMembers, G - g0);
    const int64_t qh = head * G + g0;
    __syncthreads();
    for (int i = tid; i < members * dk; i += kStepThreads) qs[i / dk][i % dk] = to_f32(q_[qh * dk + i]);
    __syncthreads();
    float o[kMembers][V];
#pragma unroll
    for (int g = 0; g < kMembers; ++g)
#pragma unroll
      for (int x = 0; x < V; ++x) o[g][x] = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int row = rg + i * groups;
      if (on && row < dk)
#pragma unroll
        for (int g = 0; g < kMembers; ++g)
          if (g < members)
#pragma unroll
            for (int x = 0; x < V; ++x) o[g][x] = fmaf(qs[g][row], s[i][x], o[g][x]);
    }
    if (on)
#pragma unroll
      for (int g = 0; g < kMembers; ++g)
        if (g < members)
#pragma unroll
          for (int x = 0; x < V; ++x) sums[(g * groups + rg) * dv + c0 + x] = o[g][x];
    __syncthreads();
    for (int i = tid; i < members * dv; i += kStepThreads) {
      const int g = i / dv, c = i - g * dv;
      float x = 0.f;
      for (int r = 0; r < groups; ++r) x += sums[(g * groups + r) * dv + c];
      y_[qh * dv + i] = from_f32<T>(x * scale);
    }
  }
}

template <typename T>
hipError_t launch(float* S, const void* q, const void* k, const void* v, const float* log_decay, void* y, int heads,
                  int H, int G, int dk, int dv, float scale, hipStream_t st) {
  const bool vec = dv % 4 == 0 && ((uintptr_t)S & 15) == 0;
  const int groups = kStepThreads / (vec ? dv / 4 : dv), rows = (dk + groups - 1) / groups;
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3(heads), dim3(kStepThreads), 0, st, S, (const T*)q, (const T*)k, (const T*)v, log_decay,
                       (T*)y, H, G, dk, dv, scale);
    return hipGetLastError();
  };
  if (vec) return rows <= 1 ? go(decay_step_kernel<T, 4, 1>) : rows <= 4 ? go(decay_step_kernel<T, 4, 4>) : go(decay_step_kernel<T, 4, 16>);
  return rows <= 4 ? go(decay_step_kernel<T, 1, 4>) : rows <= 16 ? go(decay_step_kernel<T, 1, 16>) : go(decay_step_kernel<T, 1, 64>);
}

}  // namespace

hipError_t launch_decay_step(float* S, const void* q, const void* k, const void* v, const float* log_decay, void* y,
                             bool bf16, int heads, int H, int G, int dk, int dv, float scale, hipStream_t st) {
  return bf16 ? launch<bf16_t>(S, q, k, v, log_decay, y, heads, H, G, dk, dv, scale, st)
              : launch<float>(S, q, k, v, log_decay, y, heads, H, G, dk, dv, scale, st);
}

}  // namespace sata
