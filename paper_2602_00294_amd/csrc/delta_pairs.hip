// What the pairs of a block's tokens leave for the delta rule's scans (delta_tiles.hpp): the products of its keys and
// queries, weighted by the decays, and the inverses of unit lower triangular matrices.
//
// Three waves to a block of 64 tokens of a query and key head: one for the pairs within each half, one for those
// across.  A wave forms k.k and q.k once, then for each value head the decays' sums (in 64 bits: differences
// of large sums keep their digits), the weights, and for a half the inverse, by
// forward substitution of the two 16 x 16 blocks on the diagonal, a column a lane, and -X22 A21 X11 below.
// All blocks side by side: the scans, which cannot be, have only products left.
// 128 heads x 64 blocks, d_k = 128, bfloat16: 125 us for 268 MB of rows and 250 MB of records; vector issue 43% of the
// cycles, three waves a SIMD (four, with 20 registers of each in scratch: 157).
#include <hip/hip_runtime.h>

#include "delta_tiles.hpp"

namespace sata {

namespace {

constexpr int C = 32;  // tokens of a half
constexpr int kPitch = C + 4;  // floats of a row in LDS

__device__ __forceinline__ double shuffle_up(double x, int d) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __shfl_up((uint32_t)u, d), hi = __shfl_up((uint32_t)(u >> 32), d);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// X = (I + A)^-1 for the strictly lower triangular A in LDS.
__device__ __forceinline__ void invert(const float* A, float* X) {
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
  float* const Y = X + 16;  // A21 X11 lies where zeros belong until it has been used
  product(A + 16 * kPitch, X, y);
#pragma unroll
  for (int r = 0; r < 4; ++r) Y[(4 * t4 + r) * kPitch + l15] = y[r];
  wave_lds_fence();
  product(X + 16 * kPitch + 16, Y, y);
#pragma unroll
  for (int r = 0; r < 4; ++r) X[(16 + 4 * t4 + r) * kPitch + l15] = -y[r];
  wave_lds_fence();
#pragma unroll
  for (int r = 0; r < 4; ++r) Y[(4 * t4 + r) * kPitch + l15] = 0.f;
  wave_lds_fence();
}

// A 32 x 32 matrix in LDS as operands of its rows (or its columns), entries in the order of a result's rows.
template <int PL, bool TRANSPOSED>
__device__ __forceinline__ void put_operand(const float* m, DeltaOperand* out) {
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
__global__ void __launch_bounds__(64) delta_pairs_kernel(DeltaArgs a, void* forward_, void* backward_) {
  constexpr bool BF16 = sizeof(T) == 2;
  constexpr int kPl = BF16 ? 1 : 3;
  using Forward = DeltaForward<BF16>;
  __shared__ __attribute__((aligned(16))) float A[C * kPitch], W[C * kPitch];  // (W, when read, takes the inverse)
  __shared__ double sums[kDeltaBlock];
  __shared__ float rates[kDeltaBlock];
  const int lane = threadIdx.x & 63, l31 = lane & 31, h = lane >> 5;
  const int blocks = (a.n + kDeltaBlock - 1) / kDeltaBlock, block = blockIdx.x / 3, part = blockIdx.x % 3, shared = blockIdx.y;
  const int t0 = block * kDeltaBlock, len = tokens_of(a.lengths, shared / a.Hk, a.n);
  if (t0 >= len) return;
  const int i0 = part == 0 ? 0 : C, j0 = part == 1 ? C : 0;  // the halves of queries (and later keys), and of keys
  f32x16 kk = zero16(), qk = zero16();  // of key j0 + result_row(i, h) with key and query i0 + l31
  {
    uint4 kj[2 * ND][kPl], x[2 * ND][kPl];
    auto load = [&](const void* p, int r, uint4 (&to)[2 * ND][kPl]) {
      load_own32<T, ND>((const T*)p + ((int64_t)shared * a.n + t0 + r + l31) * a.dk, t0 + r + l31 < len, a.dk, to);
    };
    load(a.k, j0, kj);
    load(a.q, i0, x);
#pragma unroll
    for (int s = 0; s < 2 * ND; ++s) qk = dot_planes32(kj[s], x[s], qk);
    if (part == 2) load(a.k, i0, x);
    else
#pragma unroll
      for (int s = 0; s < 2 * ND; ++s)
#pragma unroll
        for (int p = 0; p < kPl; ++p) x[s][p] = kj[s][p];
#pragma unroll
    for (int s = 0; s < 2 * ND; ++s) kk = dot_planes32(kj[s], x[s], kk);
    settle_mfma32();
  }
  for (int v = 0; v < a.G; ++v) {
    const int64_t head = (int64_t)shared * a.G + v, at = head * a.n + t0 + lane;
    const bool there = t0 + lane < len;
    double sum = there ? delta_rate(a.g[at]) : 0.0;
    const float beta = there ? a.beta[at] : 0.f;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const double x = shuffle_up(sum, d);
      if (lane >= d) sum += x;
    }
    wave_lds_fence();  // (the last value head's readers are done)
    sums[lane] = sum, rates[lane] = beta;
    wave_lds_fence();
    auto* const forward = (Forward*)forward_ + head * blocks + block;
    auto* const backward = (DeltaBackward*)backward_ + head * blocks + block;
    if (part == 0) {
      const double last = sums[kDeltaBlock - 1];
      const float early = (float)exp(sum), late = (float)exp(last - sum);
      const FloatPair whole = float_pair(exp(last));
      forward->early[lane] = early, forward->late[lane] = late * beta;
      if (lane == 0) forward->whole = whole;
      if constexpr (BACK) {
        backward->early[lane] = early, backward->late[lane] = late, backward->beta[lane] = beta;
        if (lane == 0) backward->whole = whole;
      }
    }
    const double my_sum = sums[i0 + l31];
    const float my_rate = rates[i0 + l31];
    float w[16], r[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int j = result_row(i, h);
      const float d = exp2_fast((float)((my_sum - sums[j0 + j]) * 1.4426950408889634));
      const bool across = part == 2;
      w[i] = across || j < l31 ? d * kk[i] : 0.f;
      r[i] = across || j <= l31 ? d * qk[i] * a.scale : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int j = result_row(i, h);
      const float beta_j = rates[j0 + j];
      A[l31 * kPitch + j] = part == 2 || j < l31 ? w[i] * beta_j : 0.f;
      W[l31 * kPitch + j] = part == 2 || j <= l31 ? r[i] * beta_j : 0.f;
    }
    wave_lds_fence();
    const int which = part == 0 ? 0 : part == 1 ? 2 : 1;
    put_operand<Forward::kPair, false>(W, forward->pairs[which]);
    if (part == 2) {
      put_operand<3, false>(A, forward->below);
    } else {
      wave_lds_fence();
      invert(A, W);
      put_operand<3, false>(W, forward->inverse[part]);
    }
    if constexpr (BACK) {
      wave_lds_fence();
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int j = result_row(i, h);
        A[l31 * kPitch + j] = part == 2 || j < l31 ? w[i] * my_rate : 0.f;
        W[l31 * kPitch + j] = r[i];
      }
      wave_lds_fence();
      put_operand<3, true>(W, backward->pairs[which]);
      if (part == 2) {
        put_operand<3, true>(A, backward->below);
      } else {
        wave_lds_fence();
        invert(A, W);
        put_operand<3, true>(W, backward->inverse[part]);
      }
    }
  }
}

template <typename T, bool BACK>
hipError_t launch(const DeltaArgs& a, void* forward, void* backward, hipStream_t s) {
  const dim3 grid((a.n + kDeltaBlock - 1) / kDeltaBlock * 3, a.heads / a.G);
  switch ((a.dk + 31) / 32) {
    case 1: hipLaunchKernelGGL((delta_pairs_kernel<T, 1, BACK>), grid, dim3(64), 0, s, a, forward, backward); break;
    case 2: hipLaunchKernelGGL((delta_pairs_kernel<T, 2, BACK>), grid, dim3(64), 0, s, a, forward, backward); break;
    case 3: hipLaunchKernelGGL((delta_pairs_kernel<T, 3, BACK>), grid, dim3(64), 0, s, a, forward, backward); break;
    default: hipLaunchKernelGGL((delta_pairs_kernel<T, 4, BACK>), grid, dim3(64), 0, s, a, forward, backward); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_pairs(const DeltaArgs& a, bool bf16, void* forward, void* backward, hipStream_t s) {
  if (backward) return bf16 ? launch<u16, true>(a, forward, backward, s) : launch<float, true>(a, forward, backward, s);
  return bf16 ? launch<u16, false>(a, forward, backward, s) : launch<float, false>(a, forward, backward, s);
}

size_t delta_forward_bytes(bool bf16, int heads, int n) {
  const size_t blocks = (size_t)heads * ((n + kDeltaBlock - 1) / kDeltaBlock);
  return blocks * (bf16 ? sizeof(DeltaForward<true>) : sizeof(DeltaForward<false>));
}

}  // namespace sata
