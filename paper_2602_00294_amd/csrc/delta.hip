// The gated delta rule: with c = 1 / sqrt(d_k), a log decay g_t and a rate beta_t for every token of a value head,
//     S' = exp(g_t) S_{t-1},   u_t = beta_t (v_t - k_t S'),   S_t = S' + k_t (x) u_t,   y_t = c q_t S_t.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "decay_power.hpp"
#include "device_common.hpp"
#include "kernels.hpp"
#include "pair_tiles.hpp"

namespace sata {

namespace {

// Token by token: a thread has a column of the state in registers, the tokens' queries and keys lie in LDS.
constexpr int kRows = 16;  // tokens staged at once

template <typename T, int ND>
__global__ void __launch_bounds__(64) delta_tokens_kernel(DeltaArgs a) {
  constexpr int kD = 32 * ND;
  __shared__ __attribute__((aligned(16))) float ks[kRows][kD], qs[kRows][kD];
  __shared__ float decays[kRows], rates[kRows];
  const int head = blockIdx.x, tid = threadIdx.x, col = blockIdx.y * 64 + tid;
  const int64_t shared = head / a.G;
  const bool on = col < a.dv;
  const int len = tokens_of(a.lengths, head / (a.Hk * a.G), a.n);
  const T* const q = (const T*)a.q + shared * a.n * a.dk;
  const T* const k = (const T*)a.k + shared * a.n * a.dk;
  const T* const v = (const T*)a.v + (int64_t)head * a.n * a.dv;
  T* const y = (T*)a.y + (int64_t)head * a.n * a.dv;
  float S[kD];
#pragma unroll
  for (int i = 0; i < kD; ++i) S[i] = a.S_in && on && i < a.dk ? a.S_in[((int64_t)head * a.dk + i) * a.dv + col] : 0.f;
  for (int t0 = 0; t0 < len; t0 += kRows) {
    const int m = min(kRows, len - t0);
    __syncthreads();
    for (int i = tid; i < m * kD; i += 64) {
      const int r = i / kD, e = i % kD;
      ks[r][e] = e < a.dk ? entry_of(k, (int64_t)(t0 + r) * a.dk + e) : 0.f;
      qs[r][e] = e < a.dk ? entry_of(q, (int64_t)(t0 + r) * a.dk + e) : 0.f;
    }
    if (tid < m) {
      decays[tid] = (float)exp(delta_rate(a.g[(int64_t)head * a.n + t0 + tid]));
      rates[tid] = a.beta[(int64_t)head * a.n + t0 + tid];
    }
    __syncthreads();
    for (int r = 0; r < m; ++r) {
      const float lam = decays[r];
      float p0 = 0.f, p1 = 0.f;
#pragma unroll
      for (int i = 0; i < kD; i += 2) {
        S[i] *= lam, S[i + 1] *= lam;
        p0 = fmaf(ks[r][i], S[i], p0), p1 = fmaf(ks[r][i + 1], S[i + 1], p1);
      }
      const float u = on ? rates[r] * (entry_of(v, (int64_t)(t0 + r) * a.dv + col) - (p0 + p1)) : 0.f;
      p0 = p1 = 0.f;
#pragma unroll
      for (int i = 0; i < kD; i += 2) {
        S[i] = fmaf(ks[r][i], u, S[i]), S[i + 1] = fmaf(ks[r][i + 1], u, S[i + 1]);
        p0 = fmaf(qs[r][i], S[i], p0), p1 = fmaf(qs[r][i + 1], S[i + 1], p1);
      }
      if (on) y[(int64_t)(t0 + r) * a.dv + col] = rounded<T>((p0 + p1) * a.scale);
    }
  }
  if (on) {
    for (int t = len; t < a.n; ++t) y[(int64_t)t * a.dv + col] = (T)0;
    if (a.S_out)
#pragma unroll
      for (int i = 0; i < kD; ++i)
        if (i < a.dk) a.S_out[((int64_t)head * a.dk + i) * a.dv + col] = S[i];
  }
}

template <typename T>
hipError_t launch_tokens(const DeltaArgs& a, hipStream_t s) {
  const dim3 grid(a.heads, (a.dv + 63) / 64);
  switch ((a.dk + 31) / 32) {
    case 1: hipLaunchKernelGGL((delta_tokens_kernel<T, 1>), grid, dim3(64), 0, s, a); break;
    case 2: hipLaunchKernelGGL((delta_tokens_kernel<T, 2>), grid, dim3(64), 0, s, a); break;
    case 3: hipLaunchKernelGGL((delta_tokens_kernel<T, 3>), grid, dim3(64), 0, s, a); break;
    default: hipLaunchKernelGGL((delta_tokens_kernel<T, 4>), grid, dim3(64), 0, s, a); break;
  }
  return hipGetLastError();
}

}  // namespace

size_t delta_prefill_scratch(bool, int, int, int, int, int) { return 0; }

hipError_t launch_delta_prefill(const DeltaArgs& a, bool bf16, void*, hipStream_t s) {
  return bf16 ? launch_tokens<u16>(a, s) : launch_tokens<float>(a, s);
}

}  // namespace sata
