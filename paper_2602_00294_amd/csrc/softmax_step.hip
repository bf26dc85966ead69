// One token of causal softmax attention over a cache: row lengths[b] of the cache becomes k
// and v, then y = sum_{s<=lengths[b]} p_s v_s with p = softmax(c q.k_s).
//
// Bound: the cache is read once, 2 (d_k + d_v) bytes a key in bfloat16.  The G query heads that share
// a key/value head are the columns of one 32 x 32 product, so a key's row serves all of
// them.  A key/value head's rows are cut into stretches for as many workgroups as keep
// every compute unit loading; a wave takes every W-th tile of 32 rows of a stretch and
// has the next tile on its way while it works, so no wave waits for another one before
// the end, where the waves' sums are joined (and the stretches' by a second kernel).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_common.hpp"
#include "kernels.hpp"
#include "pair_tiles.hpp"

namespace sata {

namespace {

constexpr int kStepWaves = 4;

// A wave's own stores to LDS before its lanes' loads.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// What a stretch (or a wave) leaves for a query head: the sums times 2^-top, scores in units of log 2.
struct StepState {
  float top, sum;
};

template <typename T, int ND>
__global__ void __launch_bounds__(64 * kStepWaves, sizeof(T) == 2 ? 2 : 1)
softmax_step_kernel(SoftmaxStepArgs a, SoftmaxStepPlan p) {
  using L = PairTile<T, ND, 32>;
  extern __shared__ __attribute__((aligned(16))) u16 smem16[];
  __shared__ StepState state[kStepWaves][32];
  const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // workgroups of one key/value head lie next to each other
  const int stretch = blockIdx.x % p.stretches, block = blockIdx.x / p.stretches % p.blocks;
  const int64_t kvh = blockIdx.x / p.stretches / p.blocks;
  const int dk = a.dk_, dv = a.dv_, at = a.lengths[kvh / a.H];
  const bool on = at >= 0 && at < a.capacity;
  const int members = min(32, a.G - 32 * block);
  const int64_t q0 = kvh * a.G + 32 * block;  // the block's first query head
  const int first = stretch * p.stretch_len, end = on ? min(at + 1, first + p.stretch_len) : 0;
  if (first >= end) {
    // (no token at all: the first stretch writes the zeros)
    if (!on && stretch == 0)
      for (int i = tid; i < members * dv; i += 64 * kStepWaves) ((T*)a.y)[q0 * dv + i] = (T)0;
    return;
  }
  T* const K = (T*)a.K + kvh * a.capacity * dk;
  T* const V = (T*)a.V + kvh * a.capacity * dv;
  const T* const kn = (const T*)a.k + kvh * dk;
  const T* const vn = (const T*)a.v + kvh * dv;
  if (block == 0 && at < first + p.stretch_len) {
    for (int i = tid; i < dk; i += 64 * kStepWaves) K[(int64_t)at * dk + i] = kn[i];
    for (int i = tid; i < dv; i += 64 * kStepWaves) V[(int64_t)at * dv + i] = vn[i];
  }
  u16* const tile = smem16 + wave * L::kElems;
  uint4 qf[2 * ND][L::kPl];
  load_own32<T, ND>((const T*)a.q + (q0 + l31) * dk, l31 < members, dk, qf);
  f32x16 o[ND];
#pragma unroll
  for (int j = 0; j < ND; ++j) o[j] = zero16();
  float top = -3.4028234e38f, sum = 0.f;
  const float c = a.scale * kLog2e;
  // (rows of the cache before the new one; that one comes from the call's k and v)
  TileStage<T, ND, 32, 64> sk, sv;
  sk.init(K, at, dk, lane);
  sv.init(V, at, dv, lane);
  auto stage = [&](const TileStage<T, ND, 32, 64>& s, int r0, const T* row, int width) {
    wave_lds_fence();
    s.put(tile, r0);
    if (at - r0 < 32) {
      wave_lds_fence();
      for (int i = lane; i < width; i += 64) TileStage<T, ND, 32, 64>::put_entry(tile + L::at(at - r0, i), row[i]);
    }
    wave_lds_fence();
  };
  constexpr int kStep = 32 * kStepWaves;
  int r0 = first + 32 * wave;
  if (r0 < end) {
    sk.fetch(r0);
    sv.fetch(r0);
  }
  for (; r0 < end; r0 += kStep) {
    stage(sk, r0, kn, dk);
    if (r0 + kStep < end) sk.fetch(r0 + kStep);
    f32x16 s = zero16();
#pragma unroll
    for (int i = 0; i < 2 * ND; ++i) {
      uint4 f[L::kPl];
      L::load_rows(tile, 0, i, f);
      s = dot_planes32(f, qf[i], s);
    }
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = r0 + result_row(i, h) > at ? -INFINITY : s[i];
      most = fmaxf(most, s[i]);
    }
    most *= c;
    stage(sv, r0, vn, dv);
    if (r0 + kStep < end) sv.fetch(r0 + kStep);
    if (__ballot(most > top + 8.f)) {
      const float next = fmaxf(top, fmaxf(most, __shfl_xor(most, 32)));
      const float keep = exp2_fast(top - next);
      top = next;
      sum *= keep;
#pragma unroll
      for (int j = 0; j < ND; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[j][i] *= keep;
    }
    float z[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      z[i] = exp2_fast(fmaf(s[i], c, -top));
      sum += z[i];
    }
    uint4 w[2][L::kPl];
    to_planes<L::kPl>(z, w);
    contract32<L, ND>(tile, 0, w, o);
  }
  settle_mfma32();
  sum += __shfl_xor(sum, 32);

  // ---- the waves' sums joined, in their order
  __syncthreads();
  float* const sums = (float*)smem16;  // [wave][member][dv]
  if (h == 0) state[wave][l31] = StepState{top, sum};
  if (l31 < members) {
    float* const row = sums + (wave * members + l31) * dv;
#pragma unroll
    for (int j = 0; j < ND; ++j)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int col = 32 * j + result_row(i, h);
        if (col < dv) row[col] = o[j][i];
      }
  }
  __syncthreads();
  for (int i = tid; i < members * dv; i += 64 * kStepWaves) {
    const int m = i / dv, col = i - m * dv;
    float most = state[0][m].top;
#pragma unroll
    for (int w = 1; w < kStepWaves; ++w) most = fmaxf(most, state[w][m].top);
    float x = 0.f, l = 0.f;
#pragma unroll
    for (int w = 0; w < kStepWaves; ++w) {
      const float k = exp2_fast(state[w][m].top - most);
      x = fmaf(sums[(w * members + m) * dv + col], k, x);
      l = fmaf(state[w][m].sum, k, l);
    }
    if (p.stretches == 1) {
      ((T*)a.y)[(q0 + m) * dv + col] = rounded<T>(x / l);
    } else {
      float* const out = a.scratch + ((q0 + m) * p.stretches + stretch) * (dv + 2);
      out[col] = x;
      if (col == 0) out[dv] = most, out[dv + 1] = l;
    }
  }
}

// The stretches' sums of one query head joined, in their order; one thread per column.
template <typename T>
__global__ void __launch_bounds__(kMaxPairDim) softmax_join_kernel(SoftmaxStepArgs a, SoftmaxStepPlan p) {
  const int64_t qh = blockIdx.x;
  const int dv = a.dv_, col = threadIdx.x, at = a.lengths[qh / a.G / a.H];
  if (col >= dv || at < 0 || at >= a.capacity) return;
  const int count = at / p.stretch_len + 1;
  const float* const in = a.scratch + qh * p.stretches * (dv + 2);
  float most = -3.4028234e38f;
  for (int s = 0; s < count; ++s) most = fmaxf(most, in[s * (dv + 2) + dv]);
  float x = 0.f, l = 0.f;
  for (int s = 0; s < count; ++s) {
    const float k = exp2_fast(in[s * (dv + 2) + dv] - most);
    x = fmaf(in[s * (dv + 2) + col], k, x);
    l = fmaf(in[s * (dv + 2) + dv + 1], k, l);
  }
  ((T*)a.y)[qh * dv + col] = rounded<T>(x / l);
}

template <typename T, int ND>
hipError_t launch_step(const SoftmaxStepArgs& a, const SoftmaxStepPlan& p, hipStream_t s) {
  // a tile for each wave; then the waves' sums
  const int bytes = std::max<int>(kStepWaves * PairTile<T, ND, 32>::kBytes,
                                  kStepWaves * std::min(32, a.G) * a.dv_ * (int)sizeof(float));
  auto kern = softmax_step_kernel<T, ND>;
  if (bytes > 64 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kern, dim3((unsigned)(a.heads * p.blocks * p.stretches)), dim3(64 * kStepWaves), bytes, s, a, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.stretches == 1) return e;
  hipLaunchKernelGGL(softmax_join_kernel<T>, dim3(a.heads * a.G), dim3((a.dv_ + 63) / 64 * 64), 0, s, a, p);
  return hipGetLastError();
}

}  // namespace

SoftmaxStepPlan plan_softmax_step(int heads, int G, int capacity, int dv) {
  SoftmaxStepPlan p;
  p.blocks = (G + 31) / 32;
  const int64_t want = std::max<int64_t>(1, 1024 / ((int64_t)heads * p.blocks));
  p.stretch_len = (int)std::max<int64_t>(256, (capacity + want * 128 - 1) / (want * 128) * 128);
  p.stretches = (capacity + p.stretch_len - 1) / p.stretch_len;
  p.bytes = p.stretches > 1 ? sizeof(float) * (size_t)heads * G * p.stretches * (dv + 2) : 0;
  return p;
}

hipError_t launch_softmax_step(const SoftmaxStepArgs& a, bool bf16, hipStream_t s) {
  const SoftmaxStepPlan p = plan_softmax_step(a.heads, a.G, a.capacity, a.dv_);
  switch ((std::max(a.dk_, a.dv_) + 31) / 32) {
    case 1: return bf16 ? launch_step<u16, 1>(a, p, s) : launch_step<float, 1>(a, p, s);
    case 2: return bf16 ? launch_step<u16, 2>(a, p, s) : launch_step<float, 2>(a, p, s);
    case 3: return bf16 ? launch_step<u16, 3>(a, p, s) : launch_step<float, 3>(a, p, s);
    default: return bf16 ? launch_step<u16, 4>(a, p, s) : launch_step<float, 4>(a, p, s);
  }
}

}  // namespace sata
