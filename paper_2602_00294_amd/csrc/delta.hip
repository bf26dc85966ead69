// The gated delta rule: with c = 1 / sqrt(d_k), a log decay g_t and a rate beta_t for every token of a value head,
//     S' = exp(g_t) S_{t-1},   u_t = beta_t (v_t - k_t S'),   S_t = S' + k_t (x) u_t,   y_t = c q_t S_t.
#include <hip/hip_runtime.h>

#include "delta_scan.hpp"
#include "delta_tiles.hpp"
#include "kernels.hpp"

namespace sata {

namespace {

template <typename T, int ND>
__global__ void __launch_bounds__(kScanThreads, 2) delta_scan_kernel(DeltaArgs a, const void* data, int slices) {
  extern __shared__ __attribute__((aligned(16))) u16 smem16[];
  delta_scan<T, ND, false>(a, data, nullptr, nullptr, blockIdx.x, slices, smem16);
}

template <typename T, int ND>
hipError_t launch_scan(const DeltaArgs& a, const void* data, hipStream_t s) {
  constexpr int bytes = DeltaLds<T, ND>::kBytes;
  auto kern = delta_scan_kernel<T, ND>;
  if (bytes > 64 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  const int slices = (a.dv + 16 * kScanWaves - 1) / (16 * kScanWaves);
  hipLaunchKernelGGL(kern, dim3(delta_grid(a.heads, slices)), dim3(kScanThreads), bytes, s, a, data, slices);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_scan_t(const DeltaArgs& a, const void* data, hipStream_t s) {
  switch ((a.dk + 31) / 32) {
    case 1: return launch_scan<T, 1>(a, data, s);
    case 2: return launch_scan<T, 2>(a, data, s);
    case 3: return launch_scan<T, 3>(a, data, s);
    default: return launch_scan<T, 4>(a, data, s);
  }
}

}  // namespace

size_t delta_prefill_scratch(bool bf16, int heads, int n) {
  return delta_forward_bytes(bf16, heads, n);
}

hipError_t launch_delta_prefill(const DeltaArgs& a, bool bf16, void* scratch, hipStream_t s) {
  if (a.n > 0) {  // (without tokens, the states alone go on)
    hipError_t e = launch_delta_pairs(a, bf16, scratch, nullptr, s);
    if (e != hipSuccess) return e;
  }
  return bf16 ? launch_scan_t<u16>(a, scratch, s) : launch_scan_t<float>(a, scratch, s);
}

}  // namespace sata
