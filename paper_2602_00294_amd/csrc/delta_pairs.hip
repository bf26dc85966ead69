// What the pairs of a chunk's tokens leave for the delta rule's scans (delta_tiles.hpp): the products of its keys and
// queries, weighted by the decays, and the inverse of a unit lower triangular matrix.
//
// A wave takes a chunk of 32 tokens of one query and key head: k.k and q.k once, then for each of its value heads the
// decays' sums (in 64 bits: differences of large sums keep their digits), the weights, and the inverse by
// forward substitution of the two 16 x 16 blocks on the diagonal, a column a lane, and
// -X22 A21 X11 below.  All chunks side by side: the scans, which cannot be, have only products left.
#include <hip/hip_runtime.h>

#include "delta_tiles.hpp"

namespace sata {

namespace {

constexpr int C = kDeltaChunk;
constexpr int kPitch = C + 4;  // floats of a row in LDS

__device__ __forceinline__ double shuffle_up(double x, int d) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __shfl_up((uint32_t)u, d), hi = __shfl_up((uint32_t)(u >> 32), d);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// X = (I + A)^-1 for the strictly lower triangular A in LDS; Y: space.
__device__ __forceinline__ void invert(const float* A, float* X, float* Y) {
  const int lane = threadIdx.x & 63, l15 = lane & 15, t4 = lane >> 4, b = 16 * (t4 & 1);
  float x[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float r = i == l15 ? 1.f : 0.f;
    const float4* const row = (const float4*)(A + (b + i) * kPitch + b);
#pragma unroll
    for (int m = 0; m < (i + 3) / 4; ++m) {
      const float4 w = row[m];
      const float f[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int y = 0; y < 4; ++y)
        if (4 * m + y < i) r = fmaf(-f[y], x[4 * m + y], r);
    }
    x[i] = i < l15 ? 0.f : r;  // (above the diagonal, whatever A holds)
  }
  if (t4 < 2) {
#pragma unroll
    for (int i = 0; i < 16; ++i) X[(b + i) * kPitch + b + l15] = x[i];
  } else if (t4 == 2) {
#pragma unroll
    for (int i = 0; i < 16; ++i) X[i * kPitch + 16 + l15] = 0.f;
  }
  wave_lds_fence();
  // rows 4 t4 .. +3, column l15 of a 16 x 16 product
  auto product = [&](const float* a, const float* c, float (&out)[4]) {
#pragma unroll
    for (int r = 0; r < 4; ++r) out[r] = 0.f;
#pragma unroll
    for (int m = 0; m < 16; m += 4) {
      float col[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) col[y] = c[(m + y) * kPitch + l15];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float4 w = *(const float4*)(a + (4 * t4 + r) * kPitch + m);
        out[r] = fmaf(w.x, col[0], fmaf(w.y, col[1], fmaf(w.z, col[2], fmaf(w.w, col[3], out[r]))));
      }
    }
  };
  float y[4];
  product(A + 16 * kPitch, X, y);  // A21 X11
#pragma unroll
  for (int r = 0; r < 4; ++r) Y[(4 * t4 + r) * kPitch + l15] = y[r];
  wave_lds_fence();
  product(X + 16 * kPitch + 16, Y, y);
#pragma unroll
  for (int r = 0; r < 4; ++r) X[(16 + 4 * t4 + r) * kPitch + l15] = -y[r];
  wave_lds_fence();
}

// A 32 x 32 matrix in LDS as operands of its rows (or its columns), entries in the order of a result's rows.
template <int PL, bool TRANSPOSED>
__device__ __forceinline__ void put_operand(const float* m, uint4 (*out)[2][64]) {
  const int lane = threadIdx.x & 63, l15 = lane & 15, t4 = lane >> 4;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = 16 * x + l15, j = 16 * (e >> 2) + 4 * t4 + (e & 3);
      v[e] = TRANSPOSED ? m[j * kPitch + i] : m[i * kPitch + j];
    }
    uint4 op[PL];
    operand_of<PL>(v, op);
#pragma unroll
    for (int p = 0; p < PL; ++p) out[p][x][lane] = op[p];
  }
}

template <typename T, int ND, bool BACK>
__global__ void __launch_bounds__(64) delta_pairs_kernel(DeltaArgs a, void* data_, void* back_) {
  constexpr bool BF16 = sizeof(T) == 2;
  constexpr int kPl = BF16 ? 1 : 3;
  __shared__ __attribute__((aligned(16))) float A[C * kPitch], X[C * kPitch], W[C * kPitch];
  __shared__ double sums[C];
  __shared__ float rates[C];
  const int lane = threadIdx.x & 63, l31 = lane & 31, h = lane >> 5;
  const int chunks = (a.n + C - 1) / C, chunk = blockIdx.x, shared = blockIdx.y, t0 = chunk * C;
  const int len = tokens_of(a.lengths, shared / a.Hk, a.n);
  if (t0 >= len) return;
  const bool there = t0 + l31 < len;
  f32x16 kk = zero16(), qk = zero16();  // of key result_row(i, h) with key and query l31
  {
    uint4 k[2 * ND][kPl], q[2 * ND][kPl];
    const int64_t row = (int64_t)shared * a.n + t0 + l31;
    load_own32<T, ND>((const T*)a.k + row * a.dk, there, a.dk, k);
    load_own32<T, ND>((const T*)a.q + row * a.dk, there, a.dk, q);
#pragma unroll
    for (int s = 0; s < 2 * ND; ++s) {
      kk = dot_planes32(k[s], k[s], kk);
      qk = dot_planes32(k[s], q[s], qk);
    }
    settle_mfma32();
  }
  for (int v = 0; v < a.G; ++v) {
    const int64_t head = (int64_t)shared * a.G + v, at = head * a.n + t0 + l31;
    double sum = there ? delta_rate(a.g[at]) : 0.0;
    const float beta = there ? a.beta[at] : 0.f;
#pragma unroll
    for (int d = 1; d < C; d *= 2) {
      const double x = shuffle_up(sum, d);
      if (l31 >= d) sum += x;
    }
    wave_lds_fence();  // (the last value head's readers are done)
    if (h == 0) sums[l31] = sum, rates[l31] = beta;
    wave_lds_fence();
    const double last = sums[C - 1];
    const float early = (float)exp(sum), late = (float)exp(last - sum), whole = (float)exp(last);
    auto* const data = (DeltaChunkData<BF16>*)data_ + head * chunks + chunk;
    float w[16], r[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int j = result_row(i, h);
      const float d = exp2_fast((float)((sum - sums[j]) * 1.4426950408889634));
      w[i] = j < l31 ? d * kk[i] : 0.f;                 // L
      r[i] = j <= l31 ? d * qk[i] * a.scale : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int j = result_row(i, h);
      A[l31 * kPitch + j] = w[i] * rates[j];
      W[l31 * kPitch + j] = j <= l31 ? r[i] * rates[j] : 0.f;
    }
    wave_lds_fence();
    put_operand<DeltaChunkData<BF16>::kPair, false>(W, data->pairs);
    wave_lds_fence();
    invert(A, X, W);
    put_operand<3, false>(X, data->inverse);
    if (h == 0) data->early[l31] = early, data->late[l31] = late * beta;
    if (lane == 0) data->whole[0] = whole;
    if constexpr (BACK) {
      auto* const back = (DeltaChunkBack<BF16>*)back_ + head * chunks + chunk;
      wave_lds_fence();
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int j = result_row(i, h);
        A[l31 * kPitch + j] = w[i] * beta;
        W[l31 * kPitch + j] = r[i];
      }
      wave_lds_fence();
      put_operand<3, true>(W, back->pairs);
      wave_lds_fence();
      invert(A, X, W);
      put_operand<3, true>(X, back->inverse);
      if (h == 0) back->early[l31] = early, back->late[l31] = late, back->beta[l31] = beta;
      if (lane == 0) back->whole[0] = whole;
    }
  }
}

template <typename T, bool BACK>
hipError_t launch(const DeltaArgs& a, void* data, void* back, hipStream_t s) {
  const dim3 grid((a.n + C - 1) / C, a.heads / a.G);
  switch ((a.dk + 31) / 32) {
    case 1: hipLaunchKernelGGL((delta_pairs_kernel<T, 1, BACK>), grid, dim3(64), 0, s, a, data, back); break;
    case 2: hipLaunchKernelGGL((delta_pairs_kernel<T, 2, BACK>), grid, dim3(64), 0, s, a, data, back); break;
    case 3: hipLaunchKernelGGL((delta_pairs_kernel<T, 3, BACK>), grid, dim3(64), 0, s, a, data, back); break;
    default: hipLaunchKernelGGL((delta_pairs_kernel<T, 4, BACK>), grid, dim3(64), 0, s, a, data, back); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_pairs(const DeltaArgs& a, bool bf16, void* data, void* back, hipStream_t s) {
  if (back) return bf16 ? launch<u16, true>(a, data, back, s) : launch<float, true>(a, data, back, s);
  return bf16 ? launch<u16, false>(a, data, back, s) : launch<float, false>(a, data, back, s);
}

size_t delta_data_bytes(bool bf16, int heads, int n) {
  const size_t chunks = (size_t)heads * ((n + C - 1) / C);
  return chunks * (bf16 ? sizeof(DeltaChunkData<true>) : sizeof(DeltaChunkData<false>));
}

}  // namespace sata
