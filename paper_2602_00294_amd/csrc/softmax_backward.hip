// Gradients of causal softmax attention, the probabilities computed again from the
// scores and lse: with c = 1 / sqrt(d_k),
//     p_ts = exp(c q_t.k_s - lse_t),  e_ts = p_ts (dy_t.v_s - delta_t),  delta_t = dy_t.y_t,
//     dq_t = c sum_{s<=t} e_ts k_s,   dk_s = c sum_{t>=s} e_ts q_t,      dv_s = sum_{t>=s} p_ts dy_t.
//
// Two launches, each sum in the registers of one wave in a fixed order:
// softmax_rows walks the keys of its queries for dq (and leaves delta),
// softmax_cols the queries of its keys, of all members of the group, for dk and dv.
// The scores and dy.v are formed in both: seven products of d columns a pair instead of five, for
// no sums of dq across workgroups.
//
// Bound: neither the matrix instructions (busy 43% of the cycles in the first, 28% in the second) nor LDS (a quarter)
// nor memory (without its loads the second took 16% less), but the chain of a tile in two waves a SIMD: loads from
// LDS, product, exponentials, barrier, loads, product.  B = 2, H = 16, n = 4096, d = 128: 596 us (577 TFLOP/s
// of the five products), the second 60% of it; 625 us without the steps that go without
// branches, where no row of the workgroup is masked.
//
// Precision: as in the forward; p and e of bfloat16 calls are rounded to bfloat16 for the
// products with dy, k and q (half a step each), float32 ones are three bfloat16 numbers.  Two numbers in bfloat16 calls:
// 595 -> 731 us of the case above, and 0.0024 -> 0.0018 off the exact gradients.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "device_common.hpp"
#include "kernels.hpp"
#include "pair_tiles.hpp"

namespace sata {

namespace {

template <typename T>
constexpr int kStaged = sizeof(T) == 2 ? 64 : 32;  // rows staged at a time

// This lane's part of the product of two rows (the other half of the lanes has the rest).
template <int ND, int PL>
__device__ __forceinline__ float dot_own(const uint4 (&a)[2 * ND][PL], const uint4 (&b)[2 * ND][PL]) {
  float r = 0.f;
#pragma unroll
  for (int s = 0; s < 2 * ND; ++s) {
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = PL - 1; i >= 0; --i) {
      const uint32_t u[4] = {a[s][i].x, a[s][i].y, a[s][i].z, a[s][i].w}, w[4] = {b[s][i].x, b[s][i].y, b[s][i].z, b[s][i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[2 * j] += lo_f32(u[j]), x[2 * j + 1] += hi_f32(u[j]);
        y[2 * j] += lo_f32(w[j]), y[2 * j + 1] += hi_f32(w[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) r = fmaf(x[j], y[j], r);
  }
  return r;
}

// A query tile's own keys row by row (see dot_row): `rows` of them from k and v on.
template <typename T, int ND, int PL>
__device__ __forceinline__ void masked_keys(const T* k, int dk, const T* v, int dv, int rows, float c, float lse,
                                            float delta, const uint4 (&qf)[2 * ND][PL], const uint4 (&df)[2 * ND][PL],
                                            f32x16 (&acc)[ND]) {
  const int l31 = threadIdx.x & 31;
#pragma unroll 1
  for (int r = 0; r < rows; ++r) {
    const float z = dot_row<T, ND>(qf, k + (int64_t)r * dk, dk);
    const float d = dot_row<T, ND>(df, v + (int64_t)r * dv, dv);
    if (r <= l31) add_row(k + (int64_t)r * dk, dk, exp2_fast(fmaf(z, c, -lse)) * (d - delta), acc);
  }
}
// Whether rows of q and dy hold a value that is not finite (for the whole wave).
template <typename T>
__device__ __forceinline__ bool rows_not_finite(const T* q, int dk, const T* dy, int dv, int rows) {
  bool bad = false;
  for (int i = threadIdx.x & 63; i < rows * dk; i += 64) bad |= !isfinite(entry_of(q, i));
  for (int i = threadIdx.x & 63; i < rows * dv; i += 64) bad |= !isfinite(entry_of(dy, i));
  return __ballot(bad) != 0;
}

template <typename T, int ND, int W>
__global__ void __launch_bounds__(64 * W, sizeof(T) == 2 ? 2 : 1) softmax_rows(SoftmaxGradArgs a, int blocks) {
  constexpr int kRows = kStaged<T>, kThreads = 64 * W;
  using L = PairTile<T, ND, kRows>;
  extern __shared__ __attribute__((aligned(16))) u16 smem16[];
  const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int qh, blk;
  if (!locate(a.heads * a.G, blocks, qh, blk)) return;
  blk = blocks - 1 - blk;  // the longest first
  const int kvh = qh / a.G, n = a.n, dk = a.dk_, dv = a.dv_;
  const int len = tokens_of(a.lengths, kvh / a.H, n);
  const int q0 = 32 * (W * blk + wave), row = q0 + l31;
  const int64_t at = (int64_t)qh * n + row;
  f32x16 acc[ND];
#pragma unroll
  for (int j = 0; j < ND; ++j) acc[j] = zero16();
  if (32 * W * blk < len) {
    uint4 qf[2 * ND][L::kPl], df[2 * ND][L::kPl];
    load_own32<T, ND>((const T*)a.y + at * dv, row < len, dv, qf);
    load_own32<T, ND>((const T*)a.dy + at * dv, row < len, dv, df);
    float delta = dot_own<ND>(qf, df);
    delta += __shfl_xor(delta, 32);
    if (row < len && h == 0) a.delta[at] = delta;
    load_own32<T, ND>((const T*)a.q + at * dk, row < len, dk, qf);
    const float c = a.scale * kLog2e, lse = row < len ? a.lse[at] * kLog2e : 0.f;
    bool odd = false;  // whether the own tile holds values that are not finite
    auto work = [&](const u16* kt, const u16* vt, int r0, bool own) {
      f32x16 s = dot_rows32<L, ND>(kt, r0, qf), d = dot_rows32<L, ND>(vt, r0, df);
      float e[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) e[i] = exp2_fast(fmaf(s[i], c, -lse)) * (d[i] - delta);
      if (own) {
        stay_in_branch();
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = result_row(i, h) > l31 ? 0.f : e[i];
        odd = tile_not_finite<L, ND>(kt, r0);
        if (odd) return;
      }
      uint4 w[2][L::kPl];
      to_planes<L::kPl>(e, w);
      contract32<L, ND>(kt, r0, w, acc);
    };
    PairStage<T, ND, kRows, kThreads> stage;
    stage.open((const T*)a.k + (int64_t)kvh * n * dk, dk, (const T*)a.v + (int64_t)kvh * n * dv, dv, len, tid);
    stage.load(smem16, 0);
    __syncthreads();
    const int steps = (min(len, 32 * W * (blk + 1)) + kRows - 1) / kRows;
    // (blocks that every query of the workgroup sees whole)
    const int all_see = 32 * W * blk / kRows;
    int st = 0;
    for (; st < all_see; ++st) {
      u16* const now = smem16 + (st & 1) * 2 * L::kElems;
      u16* const next = smem16 + ((st + 1) & 1) * 2 * L::kElems;
      stage.fetch((st + 1) * kRows);
#pragma unroll
      for (int r = 0; r < kRows; r += 32) work(now, now + L::kElems, r, false);
      stage.put(next, (st + 1) * kRows);
      __syncthreads();
    }
    for (; st < steps; ++st) {
      u16* const now = smem16 + (st & 1) * 2 * L::kElems;
      u16* const next = smem16 + ((st + 1) & 1) * 2 * L::kElems;
      stage.step(now, next, st + 1 < steps, (st + 1) * kRows, [&](const u16* buf, int r) {
        const int k0 = st * kRows + r;
        if (k0 <= q0) work(buf, buf + L::kElems, r, k0 == q0);
      });
      __syncthreads();
    }
    settle_mfma32();
    if (__builtin_expect(odd, 0)) {
      const int64_t key = (int64_t)kvh * n + q0;
      masked_keys<T, ND>((const T*)a.k + key * dk, dk, (const T*)a.v + key * dv, dv, min(32, len - q0), c, lse, delta, qf, df, acc);
    }
  }
  if (row < n) store_row32<T, ND>((T*)a.dq + at * dk, dk, acc, row < len ? a.scale : 0.f, row >= len);
}

// Rows behind the sequence are zeros of probability zero, but a key or value that is not finite makes NaN of
// them: for such keys (rare) they are taken out of a tile's weights x of rows t0 .. +31.
template <int ND, int PL>
__device__ __forceinline__ bool own_not_finite(const uint4 (&own)[2 * ND][PL]) {
  uint32_t bad = 0;
#pragma unroll
  for (int s = 0; s < 2 * ND; ++s) bad |= not_finite_bits(own[s][PL - 1]);
  return __ballot(bad != 0) != 0;
}
template <typename X>
__device__ __forceinline__ void without_padding(X& x, int t0, int len) {
  stay_in_branch();
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = t0 + result_row(i, (threadIdx.x & 63) >> 5) < len ? x[i] : 0.f;
}

// A tile of 32 keys has two waves, which share its pairs: wave t of the first half forms the scores, the
// probabilities and dv, wave t of the second dy.v, e and dk, 4 ND matrix instructions each a pair of tiles;
// the probabilities go from one to the other through LDS, in float32, behind a barrier in the
// middle of each step.
template <typename T, int ND, int W>
__global__ void __launch_bounds__(64 * W, sizeof(T) == 2 ? 2 : 1) softmax_cols(SoftmaxGradArgs a, int blocks) {
  constexpr int kRows = kStaged<T>, kThreads = 64 * W, kTiles = W / 2, kSub = kRows / 32;
  using L = PairTile<T, ND, kRows>;
  constexpr int kBuf = 2 * L::kElems + 4 * kRows;  // Q rows, dy rows, then lse and delta as float
  extern __shared__ __attribute__((aligned(16))) u16 smem16[];
  const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool for_k = wave >= kTiles;
  // this pair of waves' probabilities: 16 numbers of a lane, four at a time
  float4* const shared_p = (float4*)(smem16 + 2 * kBuf) + wave % kTiles * kSub * 4 * 64 + lane;
  int kvh, blk;
  if (!locate(a.heads, blocks, kvh, blk)) return;  // (the first keys have the longest sweeps)
  const int n = a.n, dk = a.dk_, dv = a.dv_;
  const int len = tokens_of(a.lengths, kvh / a.H, n);
  const int k0 = 32 * (kTiles * blk + wave % kTiles), row = k0 + l31;
  const int64_t at = (int64_t)kvh * n + row;
  f32x16 acc[ND];  // dv or dk
#pragma unroll
  for (int j = 0; j < ND; ++j) acc[j] = zero16();
  if (32 * kTiles * blk < len) {
    uint4 own[2 * ND][L::kPl];  // k or v
    load_own32<T, ND>(for_k ? (const T*)a.v + at * dv : (const T*)a.k + at * dk, row < len, for_k ? dv : dk, own);
    const bool strange = own_not_finite<ND>(own);
    const float c = a.scale * kLog2e;
    bool odd = false;  // whether own tiles hold values that are not finite: such a member's is left out
    PairStage<T, ND, kRows, kThreads> stage;
    const int first = 32 * kTiles * blk / kRows, steps = (len + kRows - 1) / kRows - first;
    int64_t base = 0;  // the member's first row
    auto open = [&](int g) {
      base = ((int64_t)kvh * a.G + g) * n;
      stage.open((const T*)a.q + base * dk, dk, (const T*)a.dy + base * dv, dv, len, tid);
    };
    auto stat_of = [&](int t0) {  // lse and delta of the staged rows, one or the other for each thread
      const int t = t0 + tid % kRows;
      if (tid >= 2 * kRows) return 0.f;
      // (a row behind the sequence: probability zero)
      if (tid < kRows) return t < len ? a.lse[base + t] * kLog2e : INFINITY;
      return t < len ? a.delta[base + t] : 0.f;
    };
    open(0);
    const float st0 = stat_of(first * kRows);
    stage.load(smem16, first * kRows);
    if (tid < 2 * kRows) ((float*)(smem16 + 2 * L::kElems))[tid] = st0;
    __syncthreads();
    const int total = steps * a.G;
    int u = 0, st = 0, g = 0;
    auto step = [&](auto whole) {
      constexpr bool kWhole = decltype(whole)::value;
      u16* const now = smem16 + (u & 1) * kBuf;
      u16* const then = smem16 + ((u + 1) & 1) * kBuf;
      const float* const stats = (const float*)(now + 2 * L::kElems) + 4 * h;
      const bool more = u + 1 < total;
      int next = st + 1;
      if (next == steps) next = 0;
      if (more && next == 0) open(++g);
      const float stat = more ? stat_of((first + next) * kRows) : 0.f;
      const int t0 = (first + st) * kRows;
      if (more) stage.fetch((first + next) * kRows);
      f32x16 x[kSub];  // scores, then probabilities; or dy.v, then e
#pragma unroll
      for (int r = 0; r < kSub; ++r) {
        if (!kWhole && t0 + 32 * r < k0) continue;
        x[r] = dot_rows32<L, ND>(now + (for_k ? L::kElems : 0), 32 * r, own);
        if (!for_k) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 z = *(const float4*)(stats + 32 * r + 8 * i);
            x[r][4 * i] = exp2_fast(fmaf(x[r][4 * i], c, -z.x));
            x[r][4 * i + 1] = exp2_fast(fmaf(x[r][4 * i + 1], c, -z.y));
            x[r][4 * i + 2] = exp2_fast(fmaf(x[r][4 * i + 2], c, -z.z));
            x[r][4 * i + 3] = exp2_fast(fmaf(x[r][4 * i + 3], c, -z.w));
            shared_p[(4 * r + i) * 64] = float4{x[r][4 * i], x[r][4 * i + 1], x[r][4 * i + 2], x[r][4 * i + 3]};
          }
          if (__builtin_expect(strange && t0 + 32 * r + 32 > len, 0)) {
            without_padding(x[r], t0 + 32 * r, len);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              shared_p[(4 * r + i) * 64] = float4{x[r][4 * i], x[r][4 * i + 1], x[r][4 * i + 2], x[r][4 * i + 3]};
          }
        }
      }
      settle_mfma32();
      __syncthreads();
#pragma unroll
      for (int r = 0; r < kSub; ++r) {
        if (!kWhole && t0 + 32 * r < k0) continue;
        float e[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = x[r][i];
        if (for_k) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 p = shared_p[(4 * r + i) * 64], z = *(const float4*)(stats + kRows + 32 * r + 8 * i);
            e[4 * i] = p.x * (e[4 * i] - z.x);
            e[4 * i + 1] = p.y * (e[4 * i + 1] - z.y);
            e[4 * i + 2] = p.z * (e[4 * i + 2] - z.z);
            e[4 * i + 3] = p.w * (e[4 * i + 3] - z.w);
          }
          if (__builtin_expect(strange && t0 + 32 * r + 32 > len, 0)) without_padding(e, t0 + 32 * r, len);
        }
        if (!kWhole && t0 + 32 * r == k0) {
          stay_in_branch();
#pragma unroll
          for (int i = 0; i < 16; ++i) e[i] = result_row(i, h) < l31 ? 0.f : e[i];
          if (tile_not_finite<L, ND>(now, 32 * r) || tile_not_finite<L, ND>(now + L::kElems, 32 * r)) {
            odd = true;
            continue;
          }
        }
        uint4 w[2][L::kPl];
        to_planes<L::kPl>(e, w);
        contract32<L, ND>(now + (for_k ? 0 : L::kElems), 32 * r, w, acc);
      }
      if (more) {
        stage.put(then, (first + next) * kRows);
        if (tid < 2 * kRows) ((float*)(then + 2 * L::kElems))[tid] = stat;
      }
      st = next;
      ++u;
      __syncthreads();
    };
    constexpr int kOwn = 32 * kTiles / kRows;  // steps with own tiles of the workgroup
    while (u < total) {
      for (int i = min(kOwn, steps); i > 0; --i) step(std::false_type{});
      for (int i = steps - kOwn; i > 0; --i) step(std::true_type{});
    }
    settle_mfma32();
    if (__builtin_expect(odd, 0)) {
      const int rows = min(32, len - k0);
      uint4 kf[2 * ND][L::kPl];
      load_own32<T, ND>((const T*)a.k + at * dk, row < len, dk, kf);
#pragma unroll 1
      for (int g = 0; g < a.G; ++g) {
        const int64_t t0 = ((int64_t)kvh * a.G + g) * n + k0;
        const T* const q = (const T*)a.q + t0 * dk;
        const T* const dy = (const T*)a.dy + t0 * dv;
        if (!rows_not_finite(q, dk, dy, dv, rows)) continue;
#pragma unroll 1
        for (int r = 0; r < rows; ++r) {
          const float p = exp2_fast(fmaf(dot_row<T, ND>(kf, q + r * dk, dk), c, -kLog2e * a.lse[t0 + r]));
          const float d = dot_row<T, ND>(own, dy + r * dv, for_k ? dv : 0);
          if (r < l31) continue;
          if (for_k) add_row(q + r * dk, dk, p * (d - a.delta[t0 + r]), acc);
          else add_row(dy + r * dv, dv, p, acc);
        }
      }
    }
  }
  if (row >= n) return;
  store_row32<T, ND>(for_k ? (T*)a.dk + at * dk : (T*)a.dv + at * dv, for_k ? dk : dv, acc, for_k ? a.scale : 1.f, row >= len);
}

// The same sums for calls with few workgroups (few_sweeps): one of four waves per 32 queries (keys), of
// which a wave takes every fourth tile of keys (queries), through LDS of its own, so that no wave
// waits for another one before the sums are joined.
template <typename T, int ND>
__global__ void __launch_bounds__(256, 1) softmax_rows_few(SoftmaxGradArgs a, int blocks) {
  using L = PairTile<T, ND, 32>;
  extern __shared__ __attribute__((aligned(16))) u16 smem16[];
  const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int qh, blk;
  if (!locate(a.heads * a.G, blocks, qh, blk)) return;
  blk = blocks - 1 - blk;  // the longest first
  const int kvh = qh / a.G, n = a.n, dk = a.dk_, dv = a.dv_;
  const int len = tokens_of(a.lengths, kvh / a.H, n);
  const int row = 32 * blk + l31;
  const int64_t at = (int64_t)qh * n + row;
  f32x16 acc[ND];
#pragma unroll
  for (int j = 0; j < ND; ++j) acc[j] = zero16();
  if (32 * blk < len) {
    u16* const tile = smem16 + wave * L::kElems;
    TileStage<T, ND, 32, 64> sk, sv;
    sk.init((const T*)a.k + (int64_t)kvh * n * dk, len, dk, lane);
    sv.init((const T*)a.v + (int64_t)kvh * n * dv, len, dv, lane);
    int t = wave;
    if (t <= blk) sv.fetch(32 * t), sk.fetch(32 * t);
    uint4 qf[2 * ND][L::kPl], df[2 * ND][L::kPl];
    load_own32<T, ND>((const T*)a.y + at * dv, row < len, dv, qf);
    load_own32<T, ND>((const T*)a.dy + at * dv, row < len, dv, df);
    float delta = dot_own<ND>(qf, df);
    delta += __shfl_xor(delta, 32);
    if (row < len && h == 0 && wave == 0) a.delta[at] = delta;
    load_own32<T, ND>((const T*)a.q + at * dk, row < len, dk, qf);
    const float c = a.scale * kLog2e, lse = row < len ? a.lse[at] * kLog2e : 0.f;
    bool odd = false;  // whether the own tile holds values that are not finite
    for (; t <= blk; t += 4) {
      wave_lds_fence();
      sv.put(tile, 32 * t);
      wave_lds_fence();
      if (t + 4 <= blk) sv.fetch(32 * (t + 4));
      const f32x16 d = dot_rows32<L, ND>(tile, 0, df);
      wave_lds_fence();
      sk.put(tile, 32 * t);
      wave_lds_fence();
      if (t + 4 <= blk) sk.fetch(32 * (t + 4));
      const f32x16 s = dot_rows32<L, ND>(tile, 0, qf);
      float e[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) e[i] = exp2_fast(fmaf(s[i], c, -lse)) * (d[i] - delta);
      if (t == blk) {
        stay_in_branch();
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = result_row(i, h) > l31 ? 0.f : e[i];
        odd = tile_not_finite<L, ND>(tile, 0);
        if (odd) break;
      }
      uint4 w[2][L::kPl];
      to_planes<L::kPl>(e, w);
      contract32<L, ND>(tile, 0, w, acc);
    }
    settle_mfma32();
    if (__builtin_expect(odd, 0)) {
      const int64_t key = (int64_t)kvh * n + 32 * blk;
      masked_keys<T, ND>((const T*)a.k + key * dk, dk, (const T*)a.v + key * dv, dv, min(32, len - 32 * blk), c, lse, delta,
                         qf, df, acc);
    }
  }
  float x[ND][4];
  join_waves<ND>(acc, (float4*)smem16, x);
  if (row < n) store_joined<T, ND>((T*)a.dq + at * dk, dk, x, row < len ? a.scale : 0.f, row >= len);
}

template <typename T, int ND>
__global__ void __launch_bounds__(256, 1) softmax_cols_few(SoftmaxGradArgs a, int blocks) {
  using L = PairTile<T, ND, 32>;
  extern __shared__ __attribute__((aligned(16))) u16 smem16[];
  __shared__ float stats[4][64];  // a wave's queries' lse, then delta
  const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int kvh, blk;
  if (!locate(a.heads, blocks, kvh, blk)) return;  // (the first keys have the longest sweeps)
  const int n = a.n, dk = a.dk_, dv = a.dv_;
  const int len = tokens_of(a.lengths, kvh / a.H, n);
  const int row = 32 * blk + l31;
  const int64_t at = (int64_t)kvh * n + row;
  f32x16 sum_v[ND], sum_k[ND];
#pragma unroll
  for (int j = 0; j < ND; ++j) sum_v[j] = sum_k[j] = zero16();
  if (32 * blk < len) {
    u16* const qt = smem16 + wave * 2 * L::kElems;
    u16* const yt = qt + L::kElems;
    // units of work: the members' tiles from this one on
    const int tiles = (len + 31) / 32 - blk, units = tiles * a.G;
    TileStage<T, ND, 32, 64> sq, sy;
    float stat = 0.f;
    int t0 = 0;
    auto fetch = [&](int u) {
      const int g = u / tiles;
      t0 = 32 * (blk + u - g * tiles);
      const int64_t base = ((int64_t)kvh * a.G + g) * n;
      sq.init((const T*)a.q + base * dk, len, dk, lane);
      sy.init((const T*)a.dy + base * dv, len, dv, lane);
      sq.fetch(t0);
      sy.fetch(t0);
      const int t = t0 + l31;
      // (a row behind the sequence: probability zero)
      if (h == 0) stat = t < len ? a.lse[base + t] * kLog2e : INFINITY;
      else stat = t < len ? a.delta[base + t] : 0.f;
    };
    int u = wave;
    if (u < units) fetch(u);
    uint4 kf[2 * ND][L::kPl], vf[2 * ND][L::kPl];
    load_own32<T, ND>((const T*)a.k + at * dk, row < len, dk, kf);
    load_own32<T, ND>((const T*)a.v + at * dv, row < len, dv, vf);
    const float c = a.scale * kLog2e;
    bool odd = false;  // whether own tiles hold values that are not finite: such a member's is left out
    for (; u < units; u += 4) {
      const bool own = u % tiles == 0, ends = t0 + 32 > len;
      wave_lds_fence();
      sq.put(qt, t0);
      sy.put(yt, t0);
      stats[wave][lane] = stat;
      wave_lds_fence();
      if (u + 4 < units) fetch(u + 4);
      const f32x16 s = dot_rows32<L, ND>(qt, 0, kf), d = dot_rows32<L, ND>(yt, 0, vf);
      float p[16], e[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        p[i] = exp2_fast(fmaf(s[i], c, -stats[wave][result_row(i, h)]));
        e[i] = p[i] * (d[i] - stats[wave][32 + result_row(i, h)]);
      }
      if (__builtin_expect(ends, 0)) {
        stay_in_branch();
        if (__builtin_expect(own_not_finite<ND>(kf) || own_not_finite<ND>(vf), 0)) {
          without_padding(p, len / 32 * 32, len);
          without_padding(e, len / 32 * 32, len);
        }
      }
      if (own) {
        stay_in_branch();
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          p[i] = result_row(i, h) < l31 ? 0.f : p[i];
          e[i] = result_row(i, h) < l31 ? 0.f : e[i];
        }
        if (tile_not_finite<L, ND>(qt, 0) || tile_not_finite<L, ND>(yt, 0)) {
          odd = true;
          continue;
        }
      }
      uint4 w[2][L::kPl];
      to_planes<L::kPl>(p, w);
      contract32<L, ND>(yt, 0, w, sum_v);
      to_planes<L::kPl>(e, w);
      contract32<L, ND>(qt, 0, w, sum_k);
    }
    settle_mfma32();
    if (__builtin_expect(odd, 0)) {
      const int rows = min(32, len - 32 * blk);
#pragma unroll 1
      for (int g = 0; g < a.G; ++g) {
        const int64_t t0 = ((int64_t)kvh * a.G + g) * n + 32 * blk;
        const T* const q = (const T*)a.q + t0 * dk;
        const T* const dy = (const T*)a.dy + t0 * dv;
        if (g * tiles % 4 != wave || !rows_not_finite(q, dk, dy, dv, rows)) continue;
#pragma unroll 1
        for (int r = 0; r < rows; ++r) {
          const float p = exp2_fast(fmaf(dot_row<T, ND>(kf, q + r * dk, dk), c, -kLog2e * a.lse[t0 + r]));
          const float e = p * (dot_row<T, ND>(vf, dy + r * dv, dv) - a.delta[t0 + r]);
          if (r < l31) continue;
          add_row(q + r * dk, dk, e, sum_k);
          add_row(dy + r * dv, dv, p, sum_v);
        }
      }
    }
  }
  float x[ND][4];
  join_waves<ND>(sum_k, (float4*)smem16, x);
  if (row < n) store_joined<T, ND>((T*)a.dk + at * dk, dk, x, a.scale, row >= len);
  join_waves<ND>(sum_v, (float4*)smem16, x);
  if (row < n) store_joined<T, ND>((T*)a.dv + at * dv, dv, x, 1.f, row >= len);
}

template <typename T, int ND>
hipError_t launch_rows_few(const SoftmaxGradArgs& a, hipStream_t s) {
  constexpr int bytes = std::max(4 * PairTile<T, ND, 32>::kBytes, 1024 * ND * (int)sizeof(float4));
  auto kern = softmax_rows_few<T, ND>;
  if (bytes > 64 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  const int blocks = (a.n + 31) / 32;
  hipLaunchKernelGGL(kern, dim3((unsigned)head_blocks(a.heads * a.G, blocks)), dim3(256), bytes, s, a, blocks);
  return hipGetLastError();
}

template <typename T, int ND>
hipError_t launch_cols_few(const SoftmaxGradArgs& a, hipStream_t s) {
  constexpr int bytes = std::max(8 * PairTile<T, ND, 32>::kBytes, 1024 * ND * (int)sizeof(float4));
  static_assert(bytes <= 159 * 1024, "LDS of one workgroup");
  auto kern = softmax_cols_few<T, ND>;
  if (bytes > 63 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  const int blocks = (a.n + 31) / 32;
  hipLaunchKernelGGL(kern, dim3((unsigned)head_blocks(a.heads, blocks)), dim3(256), bytes, s, a, blocks);
  return hipGetLastError();
}

template <typename T, int ND, int W>
hipError_t launch_rows(const SoftmaxGradArgs& a, hipStream_t s) {
  constexpr int bytes = 4 * PairTile<T, ND, kStaged<T>>::kBytes;
  auto kern = softmax_rows<T, ND, W>;
  if (bytes > 64 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  const int blocks = (a.n + 32 * W - 1) / (32 * W);
  hipLaunchKernelGGL(kern, dim3((unsigned)head_blocks(a.heads * a.G, blocks)), dim3(64 * W), bytes, s, a, blocks);
  return hipGetLastError();
}

template <typename T, int ND, int W>
hipError_t launch_cols(const SoftmaxGradArgs& a, hipStream_t s) {
  constexpr int bytes = 2 * (2 * PairTile<T, ND, kStaged<T>>::kBytes + 8 * kStaged<T>) + W / 2 * kStaged<T> * 128;
  static_assert(bytes <= 160 * 1024, "LDS of one workgroup");
  auto kern = softmax_cols<T, ND, W>;
  if (bytes > 64 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  const int blocks = (a.n + 16 * W - 1) / (16 * W);
  hipLaunchKernelGGL(kern, dim3((unsigned)head_blocks(a.heads, blocks)), dim3(64 * W), bytes, s, a, blocks);
  return hipGetLastError();
}

template <typename T, int ND>
hipError_t launch_backward(const SoftmaxGradArgs& a, hipStream_t s) {
  constexpr bool bf16 = sizeof(T) == 2;
  const int64_t heads = (int64_t)a.heads * a.G;
  hipError_t e = few_sweeps<T, ND>(heads, a.n)         ? launch_rows_few<T, ND>(a, s)
                 : bf16 && eight_waves(heads, a.n) ? launch_rows<T, ND, bf16 ? 8 : 4>(a, s)
                                                   : launch_rows<T, ND, 4>(a, s);
  if (e != hipSuccess) return e;
  if constexpr (bf16 || ND <= 2)  // (four waves' tiles of two wide float32 tensors, 192 KB, are more than the LDS)
    if (few_sweeps<T, ND>(a.heads, a.n)) return launch_cols_few<T, ND>(a, s);
  return launch_cols<T, ND, bf16 ? 8 : 4>(a, s);
}

}  // namespace

hipError_t launch_softmax_backward(const SoftmaxGradArgs& a, bool bf16, hipStream_t s) {
  switch ((std::max(a.dk_, a.dv_) + 31) / 32) {
    case 1: return bf16 ? launch_backward<u16, 1>(a, s) : launch_backward<float, 1>(a, s);
    case 2: return bf16 ? launch_backward<u16, 2>(a, s) : launch_backward<float, 2>(a, s);
    case 3: return bf16 ? launch_backward<u16, 3>(a, s) : launch_backward<float, 3>(a, s);
    default: return bf16 ? launch_backward<u16, 4>(a, s) : launch_backward<float, 4>(a, s);
  }
}

}  // namespace sata
