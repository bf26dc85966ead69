// One token of the gated delta rule: S' = exp(g) S, u = beta (v - k S'), S = S' + k (x) u, y = c q S.
//
// Bound: the state is read and written once, 8 d_k d_v bytes a head.  A workgroup holds a head's whole
// state in registers, a thread R rows of V columns, all loaded at once.  Both products with the state are
// formed in the same pass, before the update: y = c (q S' + (q.k) u); their rows' sums are joined in
// LDS once.  The states are streamed (nontemporal), as those of the decayed tokens.
// 2048 states of 128 x 128 (268 MB): 60.5 us, 4.5 TB/s; 16 of 64 x 64: 5.6 us.
#include <hip/hip_runtime.h>

#include "decay_power.hpp"
#include "device_common.hpp"
#include "kernels.hpp"

namespace sata {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kStepThreads = 256;

// V: columns of a thread (4: whole 16-byte vectors; 1); R: rows of a thread at most.
template <typename T, int V, int R>
__global__ void __launch_bounds__(kStepThreads) delta_step_kernel(DeltaArgs a, float* __restrict__ S_) {
  __shared__ float sums[2][kStepThreads * V];  // [of k, q][row group][column]
  __shared__ float dots[kStepThreads];         // q.k over a row group's rows
  const int64_t head = blockIdx.x, shared = head / a.G;
  const int dk = a.dk, dv = a.dv;
  const int tid = threadIdx.x, cols = dv / V, groups = kStepThreads / cols;
  const int rg = tid / cols, c0 = (tid - rg * cols) * V;
  const bool on = rg < groups;
  float* const S = S_ + head * dk * dv + c0;
  float s[R][V], k[R], q[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int row = rg + i * groups;
#pragma unroll
    for (int x = 0; x < V; ++x) s[i][x] = 0.f;
    k[i] = q[i] = 0.f;
    if (on && row < dk) {
      if constexpr (V == 4) {
        const f32x4 f = __builtin_nontemporal_load((const f32x4*)(S + row * dv));
#pragma unroll
        for (int x = 0; x < 4; ++x) s[i][x] = f[x];
      } else {
        s[i][0] = S[row * dv];
      }
      k[i] = to_f32(((const T*)a.k)[shared * dk + row]);
      q[i] = to_f32(((const T*)a.q)[shared * dk + row]);
    }
  }
  const float beta = a.beta[head];
  float w[V];
#pragma unroll
  for (int x = 0; x < V; ++x) w[x] = on ? to_f32(((const T*)a.v)[head * dv + c0 + x]) : 0.f;
  const FloatPair lam = float_pair(exp(delta_rate(a.g[head])));
  float ks[V], qs[V], qk = 0.f;
#pragma unroll
  for (int x = 0; x < V; ++x) ks[x] = qs[x] = 0.f;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int row = rg + i * groups;
    if (on && row < dk) {
#pragma unroll
      for (int x = 0; x < V; ++x) {
        s[i][x] = times(s[i][x], lam);
        ks[x] = fmaf(k[i], s[i][x], ks[x]);
        qs[x] = fmaf(q[i], s[i][x], qs[x]);
      }
      qk = fmaf(q[i], k[i], qk);
    }
  }
  if (on) {
#pragma unroll
    for (int x = 0; x < V; ++x) sums[0][rg * dv + c0 + x] = ks[x], sums[1][rg * dv + c0 + x] = qs[x];
    if (c0 == 0) dots[rg] = qk;
  }
  __syncthreads();
  if (!on) return;
#pragma unroll
  for (int x = 0; x < V; ++x) ks[x] = qs[x] = 0.f;
  qk = 0.f;
  for (int r = 0; r < groups; ++r) {
#pragma unroll
    for (int x = 0; x < V; ++x) ks[x] += sums[0][r * dv + c0 + x], qs[x] += sums[1][r * dv + c0 + x];
    qk += dots[r];
  }
#pragma unroll
  for (int x = 0; x < V; ++x) w[x] = beta * (w[x] - ks[x]);
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int row = rg + i * groups;
    if (row < dk) {
#pragma unroll
      for (int x = 0; x < V; ++x) s[i][x] = fmaf(k[i], w[x], s[i][x]);
      if constexpr (V == 4) __builtin_nontemporal_store(f32x4{s[i][0], s[i][1], s[i][2], s[i][3]}, (f32x4*)(S + row * dv));
      else S[row * dv] = s[i][0];
    }
  }
  if (rg == 0) {
#pragma unroll
    for (int x = 0; x < V; ++x) ((T*)a.y)[head * dv + c0 + x] = from_f32<T>(fmaf(qk, w[x], qs[x]) * a.scale);
  }
}

template <typename T>
hipError_t launch(const DeltaArgs& a, float* S, hipStream_t st) {
  const bool vec = a.dv % 4 == 0 && ((uintptr_t)S & 15) == 0;
  const int groups = kStepThreads / (vec ? a.dv / 4 : a.dv), rows = (a.dk + groups - 1) / groups;
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3(a.heads), dim3(kStepThreads), 0, st, a, S);
    return hipGetLastError();
  };
  if (vec) return rows <= 1 ? go(delta_step_kernel<T, 4, 1>) : rows <= 4 ? go(delta_step_kernel<T, 4, 4>) : go(delta_step_kernel<T, 4, 16>);
  return rows <= 4 ? go(delta_step_kernel<T, 1, 4>) : rows <= 16 ? go(delta_step_kernel<T, 1, 16>) : go(delta_step_kernel<T, 1, 64>);
}

}  // namespace

hipError_t launch_delta_step(const DeltaArgs& a, float* S, bool bf16, hipStream_t st) {
  return bf16 ? launch<bf16_t>(a, S, st) : launch<float>(a, S, st);
}

}  // namespace sata
