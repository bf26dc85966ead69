// One token of causal softmax attention over a cache: row lengths[b] of the cache becomes k
// and v, then y = sum_{s<=lengths[b]} p_s v_s with p = softmax(c q.k_s).
//
// Bound: the cache is read once, 2 (d_k + d_v) bytes a key in bfloat16.  The G query heads that share
// a key/value head are the columns of one 32 x 32 product, so a key's row serves all of
// them.  The heads' caches are cut into stretches of one length, which the lengths of the
// sequences decide on the card: as many of them as it holds workgroups at a time, so that
// sequences of any lengths keep every compute unit loading to the end.  (With very many sequences the
// capacity decides.)  A wave takes every
// W-th tile of 32 rows of a stretch and has the next tile on its way while it works, so no
// wave waits for another one before the end, where the waves' sums are joined (and those of
// a head of several stretches by a second kernel).
// 128 heads of d = 128 in groups of four, sequences of 1 to 8192 rows (286 MB): 56 us (5.12 TB/s; a
// copy of 4 GB 4.9), 78 with stretches of one length for all calls and plain loads; the same
// with all caches full (537 MB) 91 us (5.92 TB/s), 104; all a quarter full 31 us, 62; one
// sequence of 131072 rows 93 us, 159.
// Loads are streamed: an earlier form took 62 us with and 70 without.
//
// Precision: scores, statistics and sums are float32; a weight is two bfloat16 numbers for its product with v in
// bfloat16 calls (three in float32 ones).  With one, outputs were 0.0023 off the exact ones, relative,
// instead of 0.0017, the rounding of the outputs; the second number costs 55.7 -> 56.4 us
// of the case above, at most 5% of others.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_common.hpp"
#include "kernels.hpp"
#include "pair_tiles.hpp"
#include "softmax_stretches.hpp"

namespace sata {

namespace {

// One head's rows [first, end) of a sequence with `at` rows and its new one.
template <typename T, int ND>
__device__ __forceinline__ void step_stretch_rows(const SoftmaxStepArgs& a, int64_t kvh, int block, int at, int first, int end,
                                           float* part, u16* smem16, StepState (*state)[32]) {
  using L = PairTile<T, ND, 32>;
  constexpr int kWeight = sizeof(T) == 2 ? 2 : 3;  // numbers of a weight
  const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int dk = a.dk_, dv = a.dv_;
  const int members = min(32, a.G - 32 * block);
  const int64_t q0 = kvh * a.G + 32 * block;  // the block's first query head
  if (at < 0 || at >= a.capacity) {  // no token
    for (int i = tid; i < members * dv; i += 64 * kStepWaves) ((T*)a.y)[q0 * dv + i] = (T)0;
    return;
  }
  T* const K = (T*)a.K + kvh * a.capacity * dk;
  T* const V = (T*)a.V + kvh * a.capacity * dv;
  const T* const kn = (const T*)a.k + kvh * dk;
  const T* const vn = (const T*)a.v + kvh * dv;
  if (block == 0 && at < end) {
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
    sk.template fetch<true>(r0);
    sv.template fetch<true>(r0);
  }
  for (; r0 < end; r0 += kStep) {
    stage(sk, r0, kn, dk);
    if (r0 + kStep < end) sk.template fetch<true>(r0 + kStep);
    f32x16 s = dot_rows32<L, ND>(tile, 0, qf);
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = r0 + result_row(i, h) > at ? -INFINITY : s[i];
      most = fmaxf(most, s[i]);
    }
    most *= c;
    stage(sv, r0, vn, dv);
    if (r0 + kStep < end) sv.template fetch<true>(r0 + kStep);
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
    uint4 w[2][kWeight];
    if constexpr (kWeight == 2) to_positive_pairs(z, w);
    else to_planes<3>(z, w);
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
    if (!part) {
      ((T*)a.y)[(q0 + m) * dv + col] = rounded<T>(x / l);
    } else {
      float* const out = part + m * (dv + 2);
      out[col] = x;
      if (col == 0) out[dv] = most, out[dv + 1] = l;
    }
  }
}

template <typename T, int ND>
__global__ void __launch_bounds__(64 * kStepWaves, sizeof(T) == 2 ? 2 : 1)
softmax_step_kernel(SoftmaxStepArgs a, SoftmaxStepPlan p) {
  extern __shared__ __attribute__((aligned(16))) u16 smem16[];
  __shared__ StepState state[kStepWaves][32];
  StepPlace f;
  if (!find_stretch(a, p, f)) return;
  const int id = blockIdx.x, b = f.b, hb = f.hb, heads_of = a.H * p.blocks;
  const int head = hb / p.blocks, at = a.lengths[b], first = f.stretch * f.len * p.unit;
  const int64_t place = (int64_t)b * heads_of + hb;
  int2* const found = (int2*)a.scratch;
  float* const sums = (float*)(found + (int64_t)a.heads * p.blocks);
  if (p.bytes && f.stretch == 0 && threadIdx.x == 0) found[place] = int2{id, f.count};
  step_stretch_rows<T, ND>(a, (int64_t)b * a.H + head, hb - head * p.blocks, at, first, min(at + 1, first + f.len * p.unit),
                           f.count == 1 ? nullptr : sums + (int64_t)id * min(32, a.G) * (a.dv_ + 2), smem16, state);
}

template <typename T, int ND>
hipError_t launch_step(const SoftmaxStepArgs& a, const SoftmaxStepPlan& p, hipStream_t s) {
  // a tile for each wave; then the waves' sums
  const int bytes = std::max<int>(kStepWaves * PairTile<T, ND, 32>::kBytes,
                                  kStepWaves * std::min(32, a.G) * a.dv_ * (int)sizeof(float));
  auto kern = softmax_step_kernel<T, ND>;
  if (bytes > 63 * 1024) {  // (1 KB is static)
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kern, dim3(p.workgroups), dim3(64 * kStepWaves), bytes, s, a, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.bytes == 0) return e;
  hipLaunchKernelGGL(softmax_join_kernel<T>, dim3(a.heads * a.G), dim3((a.dv_ + 63) / 64 * 64), 0, s, a, p);
  return hipGetLastError();
}

}  // namespace

SoftmaxStepPlan plan_softmax_step(bool bf16, int heads, int H, int G, int capacity, int dv, int members, int places) {
  SoftmaxStepPlan p;
  p.members = members;
  p.blocks = (G + members - 1) / members;
  const int count = heads * p.blocks, units = (capacity + p.unit - 1) / p.unit, B = heads / H;
  p.places = places ? places : bf16 ? 512 : 256;
  if ((int64_t)count * ((units + p.least - 1) / p.least) <= p.places) {
    p.fixed_len = p.least;  // (all find a place)
  } else if (B > 384) {
    // (each workgroup reads all lengths, in steps of 64: us with stretches cut by them and by the capacity, 256 sequences
    // of 8 heads and up to 2048 rows 176 and 199, 300 of one of up to 4096 68 and 83, 1000 of one of up to 2048 112
    // and 113, 512 of 8 of up to 1024 228 and 174, 2000 of 8 of up to 256 746 and 247.  In long caches, d = 64, lengths
    // of all sizes / one sequence full among short ones: 400 of one of up to 131072 1506 / 45 and 1134 / 204, 400 of 8 of
    // up to 32768 2143 / 74 and 2454 / 108, 1000 of one of up to 16384 400 / 40 and 396 / 50, 4000 of one of up to 32768
    // 2593 / 342 and 3005 / 113: what the capacity loses where one sequence is much longer than the others it
    // gains elsewhere, and it never takes the time of the full caches)
    const int most = std::min(8, std::max(4, (4 * p.places + count - 1) / count));
    p.fixed_len = std::max(8, (units + most - 1) / most);
  }
  if (p.fixed_len) p.fixed = (units + p.fixed_len - 1) / p.fixed_len;
  p.workgroups = p.fixed ? count * p.fixed
                         : (int)std::min<int64_t>(std::max(p.places, count) + count,
                                                  (int64_t)count * ((units + p.least - 1) / p.least));
  p.bytes = p.workgroups > count
                ? sizeof(int2) * (size_t)count + sizeof(float) * (size_t)p.workgroups * std::min(members, G) * (dv + 2)
                : 0;
  return p;
}

hipError_t launch_softmax_step(const SoftmaxStepArgs& a, bool bf16, hipStream_t s) {
  const SoftmaxStepPlan p = plan_softmax_step(bf16, a.heads, a.H, a.G, a.capacity, a.dv_);
  switch ((std::max(a.dk_, a.dv_) + 31) / 32) {
    case 1: return bf16 ? launch_step<u16, 1>(a, p, s) : launch_step<float, 1>(a, p, s);
    case 2: return bf16 ? launch_step<u16, 2>(a, p, s) : launch_step<float, 2>(a, p, s);
    case 3: return bf16 ? launch_step<u16, 3>(a, p, s) : launch_step<float, 3>(a, p, s);
    default: return bf16 ? launch_step<u16, 4>(a, p, s) : launch_step<float, 4>(a, p, s);
  }
}

}  // namespace sata
