// The stretches of caches that single tokens are read in: which one a workgroup takes, and the join of their sums.
#pragma once

#include <hip/hip_runtime.h>

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

// A workgroup's stretch: of sequence b, head and block of query heads hb, the stretch-th of `count`, `len` units each.
struct StepPlace {
  int b, hb, stretch, count, len;
};
// (false: there is none)
__device__ __forceinline__ bool find_stretch(const SoftmaxStepArgs& a, const SoftmaxStepPlan& p, StepPlace& f) {
  const int id = blockIdx.x, heads_of = a.H * p.blocks;
  int b, hb, stretch, count, len = p.fixed_len;
  if (p.fixed) {
    const int place = id / p.fixed;
    stretch = id - place * p.fixed, b = place / heads_of, hb = place - b * heads_of;
    count = (step_units(a, p, b) + len - 1) / len;
    if (stretch >= count) return false;
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
    if (!here) return false;
    const int from = __builtin_ctzll(here);
    b = __builtin_amdgcn_readlane(b0, from);
    int rest = id - __builtin_amdgcn_readlane(before, from) * heads_of;
    count = (step_units(a, p, b) + len - 1) / len;
    for (; rest >= count * heads_of; count = (step_units(a, p, b) + len - 1) / len) rest -= count * heads_of, ++b;
    // (a head's stretches lie next to each other)
    hb = rest / count, stretch = rest - hb * count;
  }
  f = StepPlace{b, hb, stretch, count, len};
  return true;
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

// The sums of one query head's stretches joined, in their order; one thread per column.  (Each wave has all
// tops at once and four stretches' sums on their way: 512 query heads of up to 12
// stretches 4.6 us, where each block counting stretches and loading one sum after the other took 7.6.)
// MEANS: stretches left their means in the sums' place.
template <typename T, bool MEANS = false>
__global__ void __launch_bounds__(kMaxPairDim) softmax_join_kernel(SoftmaxStepArgs a, SoftmaxStepPlan p) {
  const int qh = blockIdx.x, kvh = qh / a.G, member = qh - kvh * a.G;
  const int dv = a.dv_, col = threadIdx.x, lane = col & 63;
  const int2* const found = (const int2*)a.scratch;
  const int2 first = found[(int64_t)kvh * p.blocks + member / p.members];  // its first stretch, and how many there are
  if (first.y == 1) return;
  const int64_t pitch = (int64_t)min(p.members, a.G) * (dv + 2);
  const float* const in = (const float*)(found + (int64_t)a.heads * p.blocks) + first.x * pitch + (member % p.members) * (dv + 2);
  float most = -3.4028234e38f;
  for (int w = lane; w < first.y; w += 64) most = fmaxf(most, in[w * pitch + dv]);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
  if constexpr (MEANS) {
    float all = 0.f, x = 0.f;
    for (int w = lane; w < first.y; w += 64) all = fmaf(in[w * pitch + dv + 1], exp2_fast(in[w * pitch + dv] - most), all);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) all += __shfl_xor(all, d);
    if (col >= dv) return;
    const float inverse = 1.f / all;
#pragma unroll 4
    for (int w = 0; w < first.y; ++w)
      x = fmaf(in[w * pitch + col], in[w * pitch + dv + 1] * exp2_fast(in[w * pitch + dv] - most) * inverse, x);
    ((T*)a.y)[(int64_t)qh * dv + col] = rounded<T>(x);
    return;
  }
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

}  // namespace

}  // namespace sata
