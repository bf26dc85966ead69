// Exact causal softmax attention: with c = 1 / sqrt(d_k),
//     lse_t = log sum_{s<=t} exp(c q_t.k_s),  p_ts = exp(c q_t.k_s - lse_t),  y_t = sum_{s<=t} p_ts v_s.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_common.hpp"
#include "kernels.hpp"
#include "pair_tiles.hpp"

namespace sata {

namespace {

// The queries' own tile row by row (see dot_row): `rows` keys and values from k and v on.
template <typename T, int ND, int PL>
__device__ __forceinline__ void masked_rows(const T* k, int dk, const T* v, int dv, int rows, float c,
                                            const uint4 (&qf)[2 * ND][PL], f32x16 (&o)[ND], float& top, float& sum) {
  const int lane = threadIdx.x & 63, l31 = lane & 31, h = lane >> 5;
#pragma unroll 1
  for (int r = 0; r < rows; ++r) {
    const float z = c * dot_row<T, ND>(qf, k + (int64_t)r * dk, dk);
    if (r > l31) continue;
    const float next = fmaxf(top, z), keep = exp2_fast(top - next), p = exp2_fast(z - next);
    top = next;
    sum = sum * keep + (h == 0 ? p : 0.f);
#pragma unroll
    for (int j = 0; j < ND; ++j)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[j][i] *= keep;
    add_row(v + (int64_t)r * dv, dv, p, o);
  }
}

// One workgroup of W waves per 32 W queries of a head, 32 to a wave, which are the columns
// of its scores and outputs; the keys are walked in tiles of 32.  The exponentials' base
// moves only when a score passes it by 2^8 (in either half of the lanes), so the outputs are rarely scaled.
//
// Bound: matrix instructions (4 ND a tile) and vector instructions (32 lanes' 16 weights: a multiply-add,
// an exponential at a quarter of the rate, a sum, a maximum, half a conversion) in equal parts:
// n = 8192, 32 heads of d = 128: 566 us (971 TFLOP/s; a large library product 1346), each busy 46% of the
// cycles.  Blocks that the whole workgroup sees go without branches, their tiles' products side
// by side: a tenth of the time less.  Half of the waves half a step behind the others: 4% more; waves of higher
// priority in their products: no change; four waves instead of eight: see eight_waves.
//
// Precision: scores, statistics and sums are float32.  A bfloat16 call's weights are rounded to
// bfloat16 for their product with v, as v's entries are (half a step each); their sum takes them
// unrounded.  As two numbers each they would take the outputs from 0.0022 off the exact ones, relative, to 0.0016, the
// rounding of the outputs, and the case above from 570 to 771 us, 16 heads of 1000 with d = 64 from 13.6 to 14.4; they
// are positive, so that nothing cancels.  float32 ones are three bfloat16 numbers each.
template <typename T, int ND, int W>
__global__ void __launch_bounds__(64 * W, sizeof(T) == 2 ? 2 : 1) softmax_prefill_kernel(SoftmaxArgs a, int blocks) {
  constexpr int kWaves = W, kThreads = 64 * W;
  constexpr int kKeys = sizeof(T) == 2 ? 64 : 32;  // keys staged at a time
  using L = PairTile<T, ND, kKeys>;
  extern __shared__ __attribute__((aligned(16))) u16 smem16[];
  const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int qh, blk;
  if (!locate(a.heads * a.G, blocks, qh, blk)) return;
  blk = blocks - 1 - blk;  // the longest first
  const int kvh = qh / a.G, n = a.n, dk = a.dk_, dv = a.dv_;
  const int len = tokens_of(a.lengths, kvh / a.H, n);
  const int q0 = 32 * (kWaves * blk + wave), row = q0 + l31;
  T* const yp = (T*)a.y + ((int64_t)qh * n + row) * dv;
  f32x16 o[ND];
#pragma unroll
  for (int j = 0; j < ND; ++j) o[j] = zero16();
  float top = -3.4028234e38f, sum = 0.f;
  const int end = min(len, 32 * kWaves * (blk + 1));  // keys that this workgroup sees
  if (32 * kWaves * blk < len) {
    uint4 qf[2 * ND][L::kPl];
    load_own32<T, ND>((const T*)a.q + ((int64_t)qh * n + row) * dk, row < len, dk, qf);
    const float c = a.scale * kLog2e;
    bool odd = false;  // whether the own tile holds values that are not finite
    // keys r0 .. +31 of a staged block; own: the queries' own tile, of which each sees its part
    auto work = [&](const u16* kt, const u16* vt, int r0, bool own) {
      f32x16 s = dot_rows32<L, ND>(kt, r0, qf);
      settle_mfma32();
      if (own) {
        stay_in_branch();
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = result_row(i, h) > l31 ? -INFINITY : s[i];
        odd = tile_not_finite<L, ND>(vt, r0);
        if (odd) return;
      }
      float most = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) most = fmaxf(most, s[i]);
      most *= c;
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
      __builtin_amdgcn_sched_barrier(0);
      uint4 w[2][L::kPl];
      to_planes<L::kPl>(z, w);
      contract32<L, ND>(vt, r0, w, o);
    };
    // a staged block that every query of the workgroup sees whole
    auto whole = [&](const u16* kt, const u16* vt) {
      constexpr int kSub = kKeys / 32;
      f32x16 s[kSub];
#pragma unroll
      for (int r = 0; r < kSub; ++r) s[r] = zero16();
#pragma unroll
      for (int i = 0; i < 2 * ND; ++i)
#pragma unroll
        for (int r = 0; r < kSub; ++r) {
          uint4 f[L::kPl];
          L::load_rows(kt, 32 * r, i, f);
          s[r] = dot_planes32(f, qf[i], s[r]);
        }
      settle_mfma32();
      float most = s[0][0];
#pragma unroll
      for (int i = 1; i < 16 * kSub; ++i) most = fmaxf(most, s[i / 16][i % 16]);
      most *= c;
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
#pragma unroll
      for (int r = 0; r < kSub; ++r) {
        float z[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          z[i] = exp2_fast(fmaf(s[r][i], c, -top));
          sum += z[i];
        }
        uint4 w[2][L::kPl];
        to_planes<L::kPl>(z, w);
        contract32<L, ND>(vt, 32 * r, w, o);
      }
    };
    PairStage<T, ND, kKeys, kThreads> stage;
    stage.open((const T*)a.k + (int64_t)kvh * n * dk, dk, (const T*)a.v + (int64_t)kvh * n * dv, dv, len, tid);
    stage.load(smem16, 0);
    __syncthreads();
    const int steps = (end + kKeys - 1) / kKeys;
    const int all_see = 32 * kWaves * blk / kKeys;
    int st = 0;
    for (; st < all_see; ++st) {
      u16* const now = smem16 + (st & 1) * 2 * L::kElems;
      u16* const next = smem16 + ((st + 1) & 1) * 2 * L::kElems;
      stage.fetch((st + 1) * kKeys);
      whole(now, now + L::kElems);
      stage.put(next, (st + 1) * kKeys);
      __syncthreads();
    }
    for (; st < steps; ++st) {
      u16* const now = smem16 + (st & 1) * 2 * L::kElems;
      u16* const next = smem16 + ((st + 1) & 1) * 2 * L::kElems;
      stage.step(now, next, st + 1 < steps, (st + 1) * kKeys, [&](const u16* buf, int r) {
        const int k0 = st * kKeys + r;
        if (k0 <= q0) work(buf, buf + L::kElems, r, k0 == q0);
      });
      __syncthreads();
    }
    settle_mfma32();
    if (__builtin_expect(odd, 0)) {
      const int64_t key = (int64_t)kvh * n + q0;
      masked_rows<T, ND>((const T*)a.k + key * dk, dk, (const T*)a.v + key * dv, dv, min(32, len - q0), c, qf, o, top, sum);
    }
  }
  if (row >= n) return;
  sum += __shfl_xor(sum, 32);
  store_row32<T, ND>(yp, dv, o, 1.f / sum, row >= len);
  if (a.lse && h == 0) a.lse[(int64_t)qh * n + row] = row < len ? top * kLn2 + logf(sum) : -INFINITY;
}

// One workgroup of four waves per 32 queries, for calls with few of them (few_sweeps): a wave takes every
// fourth tile of keys, through LDS of its own, so no wave waits for another one before the sums are joined.
// Bound: the latency of a tile's chain (loads, product, exponentials, product), about 1.2 us, times
// n / 128 of them.
template <typename T, int ND>
__global__ void __launch_bounds__(256, 1) softmax_prefill_few(SoftmaxArgs a, int blocks) {
  using L = PairTile<T, ND, 32>;
  extern __shared__ __attribute__((aligned(16))) u16 smem16[];
  __shared__ float2 state[4][32];  // a wave's exponentials' base and their sum
  const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int qh, blk;
  if (!locate(a.heads * a.G, blocks, qh, blk)) return;
  blk = blocks - 1 - blk;  // the longest first
  const int kvh = qh / a.G, n = a.n, dk = a.dk_, dv = a.dv_;
  const int len = tokens_of(a.lengths, kvh / a.H, n);
  const int row = 32 * blk + l31;
  T* const yp = (T*)a.y + ((int64_t)qh * n + row) * dv;
  float* const lse = a.lse ? a.lse + (int64_t)qh * n + row : nullptr;
  const bool last = wave == 0 && h == 0 && row < n;  // the lane that writes a row's lse
  float x[ND][4];
  if (32 * blk >= len) {
#pragma unroll
    for (int j = 0; j < ND; ++j) x[j][0] = x[j][1] = x[j][2] = x[j][3] = 0.f;
    if (row < n) store_joined<T, ND>(yp, dv, x, 0.f, true);
    if (lse && last) *lse = -INFINITY;
    return;
  }
  f32x16 o[ND];
#pragma unroll
  for (int j = 0; j < ND; ++j) o[j] = zero16();
  float top = -3.4028234e38f, sum = 0.f;
  uint4 qf[2 * ND][L::kPl];
  load_own32<T, ND>((const T*)a.q + ((int64_t)qh * n + row) * dk, row < len, dk, qf);
  const float c = a.scale * kLog2e;
  bool odd = false;  // whether the own tile holds values that are not finite
  u16* const tile = smem16 + wave * L::kElems;
  TileStage<T, ND, 32, 64> sk, sv;
  sk.init((const T*)a.k + (int64_t)kvh * n * dk, len, dk, lane);
  sv.init((const T*)a.v + (int64_t)kvh * n * dv, len, dv, lane);
  int t = wave;
  if (t <= blk) sk.fetch(32 * t), sv.fetch(32 * t);
  for (; t <= blk; t += 4) {
    wave_lds_fence();
    sk.put(tile, 32 * t);
    wave_lds_fence();
    if (t + 4 <= blk) sk.fetch(32 * (t + 4));
    f32x16 s = dot_rows32<L, ND>(tile, 0, qf);
    settle_mfma32();
    if (t == blk) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = result_row(i, h) > l31 ? -INFINITY : s[i];
    }
    float most = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) most = fmaxf(most, s[i]);
    most *= c;
    wave_lds_fence();
    sv.put(tile, 32 * t);
    wave_lds_fence();
    if (t + 4 <= blk) sv.fetch(32 * (t + 4));
    if (t == blk) {
      odd = tile_not_finite<L, ND>(tile, 0);
      if (odd) break;
    }
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
  if (__builtin_expect(odd, 0))
    masked_rows<T, ND>((const T*)a.k + ((int64_t)kvh * n + 32 * blk) * dk, dk, (const T*)a.v + ((int64_t)kvh * n + 32 * blk) * dv,
                       dv, min(32, len - 32 * blk), c, qf, o, top, sum);
  sum += __shfl_xor(sum, 32);
  if (h == 0) state[wave][l31] = float2{top, sum};
  __syncthreads();
  float most = state[0][l31].x, total = 0.f;
#pragma unroll
  for (int w = 1; w < 4; ++w) most = fmaxf(most, state[w][l31].x);
#pragma unroll
  for (int w = 0; w < 4; ++w) total = fmaf(state[w][l31].y, exp2_fast(state[w][l31].x - most), total);
  const float keep = exp2_fast(top - most);
#pragma unroll
  for (int j = 0; j < ND; ++j)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[j][i] *= keep;
  join_waves<ND>(o, (float4*)smem16, x);
  if (row >= n) return;
  store_joined<T, ND>(yp, dv, x, 1.f / total, row >= len);
  if (lse && last) *lse = row < len ? most * kLn2 + logf(total) : -INFINITY;
}

template <typename T, int ND, int W>
hipError_t launch_prefill_w(const SoftmaxArgs& a, hipStream_t s) {
  constexpr int kKeys = sizeof(T) == 2 ? 64 : 32;
  constexpr int bytes = 4 * PairTile<T, ND, kKeys>::kBytes;
  static_assert(bytes <= 160 * 1024, "LDS of one workgroup");
  auto kern = softmax_prefill_kernel<T, ND, W>;
  if (bytes > 64 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  const int blocks = (a.n + 32 * W - 1) / (32 * W);
  hipLaunchKernelGGL(kern, dim3((unsigned)head_blocks(a.heads * a.G, blocks)), dim3(64 * W), bytes, s, a, blocks);
  return hipGetLastError();
}

template <typename T, int ND>
hipError_t launch_prefill_few(const SoftmaxArgs& a, hipStream_t s) {
  constexpr int bytes = std::max(4 * PairTile<T, ND, 32>::kBytes, 1024 * ND * (int)sizeof(float4));
  auto kern = softmax_prefill_few<T, ND>;
  if (bytes > 64 * 1024 - 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  const int blocks = (a.n + 31) / 32;
  hipLaunchKernelGGL(kern, dim3((unsigned)head_blocks(a.heads * a.G, blocks)), dim3(256), bytes, s, a, blocks);
  return hipGetLastError();
}

template <typename T, int ND>
hipError_t launch_prefill(const SoftmaxArgs& a, hipStream_t s) {
  if (few_sweeps<T, ND>((int64_t)a.heads * a.G, a.n)) return launch_prefill_few<T, ND>(a, s);
  if constexpr (sizeof(T) == 2)
    if (eight_waves((int64_t)a.heads * a.G, a.n)) return launch_prefill_w<T, ND, 8>(a, s);
  return launch_prefill_w<T, ND, 4>(a, s);
}

}  // namespace

hipError_t launch_softmax_prefill(const SoftmaxArgs& a, bool bf16, hipStream_t s) {
  switch ((std::max(a.dk_, a.dv_) + 31) / 32) {
    case 1: return bf16 ? launch_prefill<u16, 1>(a, s) : launch_prefill<float, 1>(a, s);
    case 2: return bf16 ? launch_prefill<u16, 2>(a, s) : launch_prefill<float, 2>(a, s);
    case 3: return bf16 ? launch_prefill<u16, 3>(a, s) : launch_prefill<float, 3>(a, s);
    default: return bf16 ? launch_prefill<u16, 4>(a, s) : launch_prefill<float, 4>(a, s);
  }
}

}  // namespace sata
