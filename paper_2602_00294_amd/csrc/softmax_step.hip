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

namespace sata {

namespace {

constexpr int kStepWaves = 4;

// What a stretch (or a wave) leaves for a query head: the sums times 2^-top, scores in units of log 2.
struct StepState {
  float top, sum;
};

// The units of a sequence's cache: one at least, for its zeros or its new row.
__device__ __forceinline__ int step_units(const SoftmaxStepArgs& a, const SoftmaxStepPlan& p, int b) {
  const int at = a.lengths[b];
  return at >= 0 && at < a.capacity ? at / p.unit + 1 : 1;
}

__device__ __forceinline__ int wave_total(int x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
  return __builtin_amdgcn_readfirstlane(x);
}

// The length of a stretch in units, the same in every wave of a call: the units over the places of the
// card, or a little more where the sequences' last, shorter stretches need places too; with about as
// many heads as places only heads of twice the mean are cut.  There are never more than p.workgroups
// stretches: max(places, heads) of full length, and one shorter one a head.
__device__ __forceinline__ int step_stretch(const SoftmaxStepArgs& a, const SoftmaxStepPlan& p, int lane) {
  const int B = a.heads / a.H, heads_of = a.H * p.blocks, heads = a.heads * p.blocks;
  int all = 0;
  for (int b = lane; b < B; b += 64) all += step_units(a, p, b);
  all = wave_total(all) * heads_of;
  const int most = max(p.places, heads);
#pragma unroll 1
  for (int i = 0; i < 4 && heads < p.places; ++i) {
    const int places = p.places - i * heads / 4, len = max(p.least, (all + places - 1) / places);
    int count = 0;
    for (int b = lane; b < B; b += 64) count += (step_units(a, p, b) + len - 1) / len;
    if (wave_total(count) * heads_of <= p.places) return len;
  }
  return max(p.least, 2 * ((all + most - 1) / most));
}

// Weights x >= 0 as two bfloat16 numbers, 2^-15 of them off at most, both above zero where x is (from 2^-117 on): an
// infinite v times either is the same infinity (a second number below zero, or zero, would make NaN of it).  The
// first is x less 2^-9 of it, cut off; what is left is at least that 2^-9.
__device__ __forceinline__ void to_positive_pairs(const float (&x)[16], uint4 (&op)[2][2]) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    uint32_t first[4];
    float rest[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = __float_as_uint(x[8 * s + 2 * i] * (1.f - 0x1p-9f));
      const uint32_t b = __float_as_uint(x[8 * s + 2 * i + 1] * (1.f - 0x1p-9f));
      first[i] = __builtin_amdgcn_perm(b, a, 0x07060302);
      rest[2 * i] = x[8 * s + 2 * i] - __uint_as_float(a & 0xffff0000u);
      rest[2 * i + 1] = x[8 * s + 2 * i + 1] - __uint_as_float(b & 0xffff0000u);
    }
    op[s][0] = uint4{first[0], first[1], first[2], first[3]};
    op[s][1] = to_bf16(rest);
  }
}

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
  const int id = blockIdx.x, heads_of = a.H * p.blocks;
  int b, hb, stretch, count, len = p.fixed_len;
  if (p.fixed) {
    const int place = id / p.fixed;
    stretch = id - place * p.fixed, b = place / heads_of, hb = place - b * heads_of;
    count = (step_units(a, p, b) + len - 1) / len;
    if (stretch >= count) return;
  } else {
    const int lane = threadIdx.x & 63, B = a.heads / a.H;
    len = step_stretch(a, p, lane);
    // ---- which one this is: a lane counts the stretches of its own sequences
    const int per = (B + 63) / 64, b0 = min(B, lane * per), b1 = min(B, b0 + per);
    int mine = 0;
    for (int i = b0; i < b1; ++i) mine += (step_units(a, p, i) + len - 1) / len;
    int before = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int x = __shfl_up(before, d);
      if (lane >= d) before += x;
    }
    before -= mine;
    const uint64_t here = __ballot(before * heads_of <= id && id < (before + mine) * heads_of);
    if (!here) return;
    const int from = __builtin_ctzll(here);
    b = __builtin_amdgcn_readlane(b0, from);
    int rest = id - __builtin_amdgcn_readlane(before, from) * heads_of;
    count = (step_units(a, p, b) + len - 1) / len;
    for (; rest >= count * heads_of; count = (step_units(a, p, b) + len - 1) / len) rest -= count * heads_of, ++b;
    // (a head's stretches lie next to each other)
    hb = rest / count, stretch = rest - hb * count;
  }
  const int head = hb / p.blocks, at = a.lengths[b], first = stretch * len * p.unit;
  const int64_t place = (int64_t)b * heads_of + hb;
  int2* const found = (int2*)a.scratch;
  float* const sums = (float*)(found + (int64_t)a.heads * p.blocks);
  if (p.bytes && stretch == 0 && threadIdx.x == 0) found[place] = int2{id, count};
  step_stretch_rows<T, ND>(a, (int64_t)b * a.H + head, hb - head * p.blocks, at, first, min(at + 1, first + len * p.unit),
                           count == 1 ? nullptr : sums + (int64_t)id * min(32, a.G) * (a.dv_ + 2), smem16, state);
}

// The sums of one query head's stretches joined, in their order; one thread per column.  (Each wave has all
// tops at once and four stretches' sums on their way: 512 query heads of up to 12
// stretches 4.6 us, where each block counting stretches and loading one sum after the other took 7.6.)
template <typename T>
__global__ void __launch_bounds__(kMaxPairDim) softmax_join_kernel(SoftmaxStepArgs a, SoftmaxStepPlan p) {
  const int qh = blockIdx.x, kvh = qh / a.G, member = qh - kvh * a.G;
  const int dv = a.dv_, col = threadIdx.x, lane = col & 63;
  const int2* const found = (const int2*)a.scratch;
  const int2 first = found[(int64_t)kvh * p.blocks + member / 32];  // its first stretch, and how many there are
  if (first.y == 1) return;
  const int64_t pitch = (int64_t)min(32, a.G) * (dv + 2);
  const float* const in = (const float*)(found + (int64_t)a.heads * p.blocks) + first.x * pitch + (member % 32) * (dv + 2);
  float most = -3.4028234e38f;
  for (int w = lane; w < first.y; w += 64) most = fmaxf(most, in[w * pitch + dv]);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
  if (col >= dv) return;
  float x = 0.f, l = 0.f;
#pragma unroll 4
  for (int w = 0; w < first.y; ++w) {
    const float k = exp2_fast(in[w * pitch + dv] - most);
    x = fmaf(in[w * pitch + col], k, x);
    l = fmaf(in[w * pitch + dv + 1], k, l);
  }
  ((T*)a.y)[(int64_t)qh * dv + col] = rounded<T>(x / l);
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

SoftmaxStepPlan plan_softmax_step(bool bf16, int heads, int H, int G, int capacity, int dv) {
  SoftmaxStepPlan p;
  p.blocks = (G + 31) / 32;
  const int count = heads * p.blocks, units = (capacity + p.unit - 1) / p.unit, B = heads / H;
  p.places = bf16 ? 512 : 256;
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
                ? sizeof(int2) * (size_t)count + sizeof(float) * (size_t)p.workgroups * std::min(32, G) * (dv + 2)
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
