// One token of causal softmax attention over caches of 4 bits an entry (packed_rows.hpp): row lengths[b] of the
// caches becomes k and v in those bits, then y = sum_{s<=lengths[b]} p_s v_s with p = softmax(c q.k_s), k_s and v_s
// being what the caches' rows stand for.
//
// Rows are never unpacked into numbers of their own.  A bfloat16 with the code's four bits as the last of its
// fraction, 0x4300 | code, is 128 + code, exactly, so two codes become operands of a product by a shift (half of them) and
// one and-or.  With s and m a group's scale and least value, X the sums over such operands, o = 128,
//     q.k_t = sum_g s_tg X_tg + (m_tg - o s_tg) (sum of q's entries in g),   X_tg = sum_i (o + code_ti) q_i
//     y     = sum_t (p_t s_tg) (o + code_tj) - sum_t (p_t s_tg) (o + 8) + sum_t p_t (m_tg + 8 s_tg),
// the second sum by products of the very operands that enter the first, product by product: a weight's rounding, 2^-18 of it in
// bfloat16 calls, counts as often as code - 8 says, not o times as well (2 us of the time below), and m + 8 s, the middle of a
// group, is no larger than its values, where sums of least values would have to cancel with sums of codes.
// What the offset takes from the scores, seven bits of 24, bfloat16 calls do not feel; float32 calls take
// 0x4180 | code << 3, o = 16, for a shift more, and take o + 8 off their scores in the same way.
// Products are v_mfma_f32_16x16x32_bf16 with the query heads of a group as columns: of keys a group of 32 entries
// at a time, rows being 16 tokens; of values 16 columns at a time over 32 tokens.  A lane reads of a key's row the bytes of
// four a (packed_rows.hpp), of a value's row those of one; scores' tokens, four a lane, are the
// weights' places in the second product, so they never leave their lanes.  Scales go through LDS: a lane needs eight
// tokens' and reads one's or two's.
//
// Bound: the cache is read once, 5 (d_k + d_v) / 8 bytes a key.
//
// Precision: codes and scales are exact operands; middles, scores, statistics and sums are float32; a weight times a
// scale is two bfloat16 numbers in bfloat16 calls, three in float32 ones.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "delta_tiles.hpp"
#include "device_common.hpp"
#include "kernels.hpp"
#include "packed_rows.hpp"
#include "pair_tiles.hpp"
#include "softmax_stretches.hpp"

namespace sata {

namespace {

// Workgroups of a CU.  Waves wait for loads more than they compute; the scheduling barriers below keep a tile's
// parts apart so that three bfloat16 workgroups have registers enough (168 each, 15 of d_k = d_v = 128 in scratch).
// 16 sequences, 8 key heads, caches of 16384 rows of 128 entries, ragged, step and join: 58.2 us with three, 60.1 with two,
// without the barriers 74 with three.  A float32 call's third plane takes the room of one.
template <typename T>
constexpr int kAtOnce = sizeof(T) == 2 ? 3 : 2;

// G bytes for each of four a, as they lie in a key's row.
template <int G>
struct KeyCodes {
  uint32_t w[G];
};
template <int G>
__device__ __forceinline__ KeyCodes<G> load_key(const uint8_t* p) {
  KeyCodes<G> c;
  if constexpr (G == 4) {
    const uint4 x = *(const uint4*)p;
    c.w[0] = x.x, c.w[1] = x.y, c.w[2] = x.z, c.w[3] = x.w;
  } else if constexpr (G == 2) {
    const uint2 x = *(const uint2*)p;
    c.w[0] = x.x, c.w[1] = x.y;
  } else {
    c.w[0] = *(const uint32_t*)p;
  }
  return c;
}
// a row's scales and least values
template <int G>
__device__ __forceinline__ KeyCodes<G> load_params(const uint8_t* row) {
  return load_key<G>(row + 16 * G);
}

// Bytes `g` of four a's, two at a time in the low bytes of the halves of a dword.
template <int G>
__device__ __forceinline__ void group_bytes(const KeyCodes<G>& c, int g, uint32_t& first, uint32_t& second) {
  if constexpr (G == 4) {
    const uint32_t sel = 0x0c000c04u + 0x00010001u * g;  // byte g of the second and of the first
    first = __builtin_amdgcn_perm(c.w[0], c.w[1], sel);
    second = __builtin_amdgcn_perm(c.w[2], c.w[3], sel);
  } else if constexpr (G == 2) {
    first = g ? (c.w[0] >> 8) & 0x00ff00ffu : c.w[0] & 0x00ff00ffu;
    second = g ? (c.w[1] >> 8) & 0x00ff00ffu : c.w[1] & 0x00ff00ffu;
  } else {
    first = __builtin_amdgcn_perm(0u, c.w[0], 0x0c010c00u);
    second = __builtin_amdgcn_perm(0u, c.w[0], 0x0c030c02u);
  }
}
// What codes count from, and the code in bits 0..3 (or 4..7) of each half as that much more.  (Both constants in registers:
// one instruction.)
template <typename T>
struct Codes {
  static constexpr float kOffset = sizeof(T) == 2 ? 128.f : 16.f;
  uint32_t mask = sizeof(T) == 2 ? 0x000f000fu : 0x00780078u, tag = sizeof(T) == 2 ? 0x43004300u : 0x41804180u;
  uint32_t less = sizeof(T) == 2 ? 0xc308c308u : 0xc1c0c1c0u;  // -(kOffset + 8), twice
  __device__ __forceinline__ Codes() { asm("" : "+v"(mask), "+v"(tag), "+v"(less)); }
  __device__ __forceinline__ uint32_t low(uint32_t x) const { return ((sizeof(T) == 2 ? x : x << 3) & mask) | tag; }
  __device__ __forceinline__ uint32_t high(uint32_t x) const { return ((sizeof(T) == 2 ? x >> 4 : x >> 1) & mask) | tag; }
};

// Entries go up to 2^120 (packed_rows.hpp), and sums over (o + code) q or weights are larger than what is left of them, by
// (o + 15) / 7.5 at most, a score's by twice that.
// Queries enter 2^8 times smaller: where a query's and a key's entries have a product at all, so have these.
// Sums over 2^21 rows of weights up to 2^8 hold scales and middles of up to 2^88; from the first larger
// ones on, a wave takes all 2^32 times smaller.  (Means of stretches, not sums, are joined.)
constexpr float kSmaller = 0x1p-8f, kFar = 0x1p88f, kFarSmaller = 0x1p-32f;

// N floats of LDS
template <int N>
struct Floats {
  float f[N];
};
template <int N>
__device__ __forceinline__ Floats<N> load_floats(const float* p) {
  Floats<N> x;
  if constexpr (N == 4) {
    const float4 v = *(const float4*)p;
    x.f[0] = v.x, x.f[1] = v.y, x.f[2] = v.z, x.f[3] = v.w;
  } else if constexpr (N == 2) {
    const float2 v = *(const float2*)p;
    x.f[0] = v.x, x.f[1] = v.y;
  } else {
    x.f[0] = *p;
  }
  return x;
}
template <int N>
__device__ __forceinline__ void store_floats(float* p, const float (&x)[N]) {
  if constexpr (N == 4) *(float4*)p = float4{x[0], x[1], x[2], x[3]};
  else if constexpr (N == 2) *(float2*)p = float2{x[0], x[1]};
  else *p = x[0];
}

// A cache of rows of 20 G bytes, read at a lane's offset from a row that is the same for the wave.
template <int G>
struct RowReader {
  static constexpr int kRow = 20 * G;
  __amdgpu_buffer_rsrc_t rsrc;
  __device__ __forceinline__ RowReader(const uint8_t* p, int rows)
      : rsrc(__builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, rows * kRow, 0x00020000)) {}
  __device__ __forceinline__ KeyCodes<G> dwords(int offset, int row) const {
    typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
    typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
    KeyCodes<G> c;
    if constexpr (G == 4) {
      const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(rsrc, offset, row * kRow, 0);
      c.w[0] = x.x, c.w[1] = x.y, c.w[2] = x.z, c.w[3] = x.w;
    } else if constexpr (G == 2) {
      const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(rsrc, offset, row * kRow, 0);
      c.w[0] = x.x, c.w[1] = x.y;
    } else {
      c.w[0] = __builtin_amdgcn_raw_buffer_load_b32(rsrc, offset, row * kRow, 0);
    }
    return c;
  }
  // the G bytes of one a
  __device__ __forceinline__ uint32_t bytes(int offset, int row) const {
    if constexpr (G == 4) return __builtin_amdgcn_raw_buffer_load_b32(rsrc, offset, row * kRow, 0);
    else if constexpr (G == 2) return (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rsrc, offset, row * kRow, 0);
    else return (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(rsrc, offset, row * kRow, 0);
  }
};

// A lane's part of 32 rows: codes and parameters of keys 16 x + l15, codes of values 4 t4 + i and 16 + 4 t4 + i,
// parameters of value l31.
template <int GK, int GV>
struct PackedTile {
  KeyCodes<GK> kc[2], kp[2];
  uint32_t vc[8];
  KeyCodes<GV> vp;
  // rows r0 .. r0 + 31, all before the last one
  __device__ __forceinline__ void load_keys(const RowReader<GK>& K, int r0) {
    const int lane = threadIdx.x & 63, l15 = lane & 15, t4 = lane >> 4;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      kc[x] = K.dwords(l15 * (20 * GK) + 4 * GK * t4 + 16 * x * (20 * GK), r0);
      kp[x] = K.dwords(l15 * (20 * GK) + 16 * GK + 16 * x * (20 * GK), r0);
    }
  }
  __device__ __forceinline__ void load_values(const RowReader<GV>& V, int r0) {
    const int lane = threadIdx.x & 63, l15 = lane & 15, t4 = lane >> 4, l31 = lane & 31;
#pragma unroll
    for (int i = 0; i < 8; ++i) vc[i] = V.bytes(4 * t4 * (20 * GV) + l15 * GV + (16 * (i >> 2) + (i & 3)) * (20 * GV), r0);
    vp = V.dwords(l31 * (20 * GV) + 16 * GV, r0);
  }
  // The same where row `at` is the last: rows behind it are read as that one, which others may be writing and which lies in
  // LDS (`fresh`, the value's 80 bytes on).
  __device__ __forceinline__ void load_last_keys(const RowReader<GK>& K, int r0, int at, const uint8_t* fresh) {
    const int lane = threadIdx.x & 63, l15 = lane & 15, t4 = lane >> 4;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int r = 16 * x + l15, row = min(r, at - r0) * (20 * GK);
      kc[x] = K.dwords(row + 4 * GK * t4, r0);
      kp[x] = K.dwords(row + 16 * GK, r0);
      if (r0 + r >= at) kc[x] = load_key<GK>(fresh + 4 * GK * t4), kp[x] = load_params<GK>(fresh);
    }
  }
  __device__ __forceinline__ void load_last_values(const RowReader<GV>& V, int r0, int at, const uint8_t* fresh) {
    const int lane = threadIdx.x & 63, l15 = lane & 15, t4 = lane >> 4, l31 = lane & 31;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = 4 * t4 + 16 * (i >> 2) + (i & 3);
      vc[i] = V.bytes(min(r, at - r0) * (20 * GV) + l15 * GV, r0);
      if (r0 + r >= at) vc[i] = load_packed<GV>(fresh + 80, l15);
    }
    vp = V.dwords(min(l31, at - r0) * (20 * GV) + 16 * GV, r0);
    if (r0 + l31 >= at) vp = load_params<GV>(fresh + 80);
  }
};

// GK, GV: groups of keys and values.
template <typename T, int GK, int GV>
__device__ __forceinline__ void packed_stretch_rows(const SoftmaxStepArgs& a, int64_t kvh, int block, int at, int first, int end,
                                                    float* part, float* sums, StepState (*state)[kPackedMembers],
                                                    uint8_t* fresh, float* scales) {
  constexpr int kPl = sizeof(T) == 4 ? 3 : 1;    // numbers of a query's entry
  constexpr int kWeight = sizeof(T) == 4 ? 3 : 2;  // of a weight
  constexpr bool kExact = sizeof(T) == 4;
  constexpr int kKey = 20 * GK, kValue = 20 * GV, kThreads = 64 * kStepWaves;
  const int tid = threadIdx.x, lane = tid & 63, l15 = lane & 15, t4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int dk = a.dk_, dv = a.dv_;
  const int members = min(kPackedMembers, a.G - kPackedMembers * block);
  const int64_t q0 = kvh * a.G + kPackedMembers * block;  // the block's first query head
  if (at < 0 || at >= a.capacity) {  // no token
    for (int i = tid; i < members * dv; i += kThreads) ((T*)a.y)[q0 * dv + i] = (T)0;
    return;
  }
  uint8_t* const K = (uint8_t*)a.K + kvh * a.capacity * kKey;
  uint8_t* const V = (uint8_t*)a.V + kvh * a.capacity * kValue;
  // ---- the new row, in LDS for this workgroup (whoever writes the cache's) and in the cache
  if (at < end) {
    if (wave == 0) {
      const bool key = lane < 16;
      if (lane < 32) {
        if (key) {
          uint32_t params[GK];
          const T* const x = (const T*)a.k + kvh * dk;
          const uint32_t codes = pack_row<GK>(l15, dk, [&](int e) { return entry_of(x, e); }, params);
          store_packed<GK>(fresh, l15, codes, params);
          if (block == 0) store_packed<GK>(K + (int64_t)at * kKey, l15, codes, params);
        } else {
          uint32_t params[GV];
          const T* const x = (const T*)a.v + kvh * dv;
          const uint32_t codes = pack_row<GV>(l15, dv, [&](int e) { return entry_of(x, e); }, params);
          store_packed<GV>(fresh + 80, l15, codes, params);
          if (block == 0) store_packed<GV>(V + (int64_t)at * kValue, l15, codes, params);
        }
      }
    }
    __syncthreads();
  }
  // ---- the query heads: operands of entries 32 g + 4 t4 .. +3 and 32 g + 16 + 4 t4 .. +3, in the codes' order, and
  // the sums over the groups as three bfloat16 numbers, one in each of the first three fours of
  // lanes
  uint4 qf[GK][kPl], qsum;
  {
    const T* const q = (const T*)a.q + (q0 + l15) * dk;
    float total[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int g = 0; g < GK; ++g) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // (dwords in the order of the products' operands: low codes of a = 0, 1, then of 2, 3, then the high ones)
        const int e = 32 * g + 4 * t4 + (i & 3) + 16 * (i >> 2);
        x[i] = l15 < members && e < dk ? kSmaller * entry_of(q, e) : 0.f;
        total[g] += x[i];
      }
      total[g] += __shfl_xor(total[g], 16);
      total[g] += __shfl_xor(total[g], 32);
      uint4 w[1][kPl];
      to_planes<kPl>(x, w);
#pragma unroll
      for (int p = 0; p < kPl; ++p) qf[g][p] = w[0][p];
    }
    float x[8];
#pragma unroll
    for (int g = 0; g < 4; ++g) x[2 * g] = g < GK ? (kExact ? 8.f : -Codes<T>::kOffset) * total[g] : 0.f, x[2 * g + 1] = g < GK ? total[g] : 0.f;
    uint4 w[1][3];
    to_planes<3>(x, w);
    qsum = t4 == 0 ? w[0][0] : t4 == 1 ? w[0][1] : t4 == 2 ? w[0][2] : uint4{0u, 0u, 0u, 0u};
  }
  f32x4 o[2 * GV];
  float base[GV];
#pragma unroll
  for (int j = 0; j < 2 * GV; ++j) o[j] = zero4();
#pragma unroll
  for (int g = 0; g < GV; ++g) base[g] = 0.f;
  float top = -3.4028234e38f, sum = 0.f;
  float smaller = 1.f;  // what values enter the sums with, the same for the wave
  const float c = a.scale * (kLog2e / kSmaller);
  constexpr int kStep = 32 * kStepWaves;
  const Codes<T> codes;
  const uint4 less = {codes.less, codes.less, codes.less, codes.less};
  // this wave's: scales of keys [32][GK], of values [32][GV], and the middles of their groups
  float* const kscale = scales + wave * 32 * (GK + 2 * GV);
  float* const vscale = kscale + 32 * GK;
  float* const vmiddle = vscale + 32 * GV;
  PackedTile<GK, GV> tile;
  const RowReader<GK> keys(K, a.capacity);
  const RowReader<GV> values(V, a.capacity);
  auto load_keys = [&](int r0) {
    if (r0 + 32 <= at) tile.load_keys(keys, r0);
    else tile.load_last_keys(keys, r0, at, fresh);
  };
  auto load_values = [&](int r0) {
    if (r0 + 32 <= at) tile.load_values(values, r0);
    else tile.load_last_values(values, r0, at, fresh);
  };
  int r0 = first + 32 * wave;
  if (r0 < end) {
    load_keys(r0);
    load_values(r0);
  }
#pragma unroll 1
  for (; r0 < end; r0 += kStep) {
    wave_lds_fence();  // (the last tile's scales have been read)
    float vs[GV], middle[GV], far = 0.f;
#pragma unroll
    for (int g = 0; g < GV; ++g) {
      vs[g] = lo_f32(tile.vp.w[g]);
      middle[g] = fmaf(8.f, vs[g], hi_f32(tile.vp.w[g]));
      far = fmaxf(far, fmaxf(vs[g], fabsf(middle[g])));
    }
    if (__builtin_expect(smaller != 1.f || __ballot(far > kFar) != 0, 0)) {
      stay_in_branch();
      if (smaller == 1.f) {
        smaller = kFarSmaller;
        settle_mfma();
#pragma unroll
        for (int j = 0; j < 2 * GV; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[j][i] *= smaller;
#pragma unroll
        for (int g = 0; g < GV; ++g) base[g] *= smaller;
      }
#pragma unroll
      for (int g = 0; g < GV; ++g) vs[g] *= smaller, middle[g] *= smaller;
    }
    if (t4 < 2) {
      float k[GK];
#pragma unroll
      for (int g = 0; g < GK; ++g) k[g] = lo_f32(t4 ? tile.kp[1].w[g] : tile.kp[0].w[g]);
      store_floats<GK>(kscale + lane * GK, k);
      store_floats<GV>(vscale + lane * GV, vs);
      store_floats<GV>(vmiddle + lane * GV, middle);
    }
    wave_lds_fence();
    // ---- scores of tokens 4 t4 .. +3 and 16 + 4 t4 .. +3 with query head l15
    float s[8];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      __builtin_amdgcn_sched_barrier(0);
      uint4 m = {0u, 0u, 0u, 0u};
      m.x = tile.kp[x].w[0];
      if constexpr (GK >= 2) m.y = tile.kp[x].w[1];
      if constexpr (GK == 4) m.z = tile.kp[x].w[2], m.w = tile.kp[x].w[3];
      f32x4 score = mfma_bf16(m, qsum, zero4()), acc[GK];
#pragma unroll
      for (int g = 0; g < GK; ++g) {
        uint32_t u, w;
        group_bytes<GK>(tile.kc[x], g, u, w);
        const uint4 e = {codes.low(u), codes.low(w), codes.high(u), codes.high(w)};
        acc[g] = zero4();
#pragma unroll
        for (int p = 0; p < kPl; ++p) {
          if constexpr (kExact) acc[g] = mfma_bf16(less, qf[g][p], acc[g]);
          acc[g] = mfma_bf16(e, qf[g][p], acc[g]);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const Floats<GK> scale = load_floats<GK>(kscale + (16 * x + 4 * t4 + i) * GK);
        s[4 * x + i] = score[i];
#pragma unroll
        for (int g = 0; g < GK; ++g) s[4 * x + i] = fmaf(scale.f[g], acc[g][i], s[4 * x + i]);
        s[4 * x + i] *= c;  // (rounded before the largest is taken off: what is left of two sizes of 10^10 is no small number)
      }
    }
    if (at < r0 + 31) {
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] = r0 + 4 * t4 + 16 * (i >> 2) + (i & 3) > at ? -INFINITY : s[i];
    }
    if (r0 + kStep < end) load_keys(r0 + kStep);
    float most = s[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) most = fmaxf(most, s[i]);
    if (__ballot(most > top + 8.f)) {
      float next = fmaxf(most, __shfl_xor(most, 16));
      next = fmaxf(top, fmaxf(next, __shfl_xor(next, 32)));
      const float keep = exp2_fast(top - next);
      top = next;
      sum *= keep;
#pragma unroll
      for (int j = 0; j < 2 * GV; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[j][i] *= keep;
#pragma unroll
      for (int g = 0; g < GV; ++g) base[g] *= keep;
    }
    // ---- weights, times the scales, and the values
    __builtin_amdgcn_sched_barrier(0);
    uint32_t pairs[4][2];  // bytes of tokens 2 i and 2 i + 1, groups 0, 1 and 2, 3
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      pairs[i][0] = __builtin_amdgcn_perm(tile.vc[2 * i + 1], tile.vc[2 * i], 0x05040100);
      pairs[i][1] = __builtin_amdgcn_perm(tile.vc[2 * i + 1], tile.vc[2 * i], 0x07060302);
    }
    if (r0 + kStep < end) load_values(r0 + kStep);
    float z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      z[i] = exp2_fast(s[i] - top);
      sum += z[i];
    }
    constexpr int kAt = GV < 2 ? GV : 2;  // groups at a time
#pragma unroll
    for (int g0 = 0; g0 < GV; g0 += kAt) {
      __builtin_amdgcn_sched_barrier(0);
      float y[kAt][8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int row = (4 * t4 + 16 * (i >> 2) + (i & 3)) * GV + g0;
        const Floats<kAt> scale = load_floats<kAt>(vscale + row), middle = load_floats<kAt>(vmiddle + row);
#pragma unroll
        for (int g = 0; g < kAt; ++g) {
          y[g][i] = z[i] * scale.f[g];
          base[g0 + g] = fmaf(z[i], middle.f[g], base[g0 + g]);
        }
      }
#pragma unroll
      for (int g = 0; g < kAt; ++g) {
        uint4 w[kWeight];
        operand_of<kWeight>(y[g], w);
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = g & 1 ? pairs[i][g0 >> 1] >> 8 : pairs[i][g0 >> 1];
          lo[i] = codes.low(x), hi[i] = codes.high(x);
        }
        f32x4 &o0 = o[2 * (g0 + g)], &o1 = o[2 * (g0 + g) + 1];
        f32x4 a0 = kExact ? zero4() : o0, a1 = kExact ? zero4() : o1;
#pragma unroll
        for (int p = 0; p < kWeight; ++p) {
          a0 = mfma_bf16(less, w[p], a0);
          a1 = mfma_bf16(less, w[p], a1);
          a0 = mfma_bf16(uint4{lo[0], lo[1], lo[2], lo[3]}, w[p], a0);
          a1 = mfma_bf16(uint4{hi[0], hi[1], hi[2], hi[3]}, w[p], a1);
        }
        if constexpr (kExact) {
#pragma unroll
          for (int i = 0; i < 4; ++i) o0[i] += a0[i], o1[i] += a1[i];
        } else {
          o0 = a0, o1 = a1;
        }
      }
    }
  }
  settle_mfma32();
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
#pragma unroll
  for (int g = 0; g < GV; ++g) {
    base[g] += __shfl_xor(base[g], 16);
    base[g] += __shfl_xor(base[g], 32);
  }

  // ---- the waves' means joined, in their order, each with its part of the weights (sums of the largest values would
  // not be numbers)
  if (t4 == 0) state[wave][l15] = StepState{top, sum};
  if (l15 < members) {
    float* const row = sums + (wave * members + l15) * dv;
    const float inverse = sum == 0.f ? 0.f : 1.f / sum / smaller;  // (0: a wave without rows)
#pragma unroll
    for (int j = 0; j < 2 * GV; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int col = 16 * j + 4 * t4 + i;
        if (col < dv) row[col] = (o[j][i] + base[j / 2]) * inverse;
      }
  }
  __syncthreads();
  for (int i = tid; i < members * dv; i += kThreads) {
    const int m = i / dv, col = i - m * dv;
    float most = state[0][m].top;
#pragma unroll
    for (int w = 1; w < kStepWaves; ++w) most = fmaxf(most, state[w][m].top);
    float x = 0.f, l = 0.f, k[kStepWaves];
#pragma unroll
    for (int w = 0; w < kStepWaves; ++w) {
      k[w] = state[w][m].sum * exp2_fast(state[w][m].top - most);
      l += k[w];
    }
    const float inverse = 1.f / l;
#pragma unroll
    for (int w = 0; w < kStepWaves; ++w) x = fmaf(sums[(w * members + m) * dv + col], k[w] * inverse, x);
    if (!part) {
      ((T*)a.y)[(q0 + m) * dv + col] = rounded<T>(x);
    } else {
      float* const out = part + m * (dv + 2);
      out[col] = x;
      if (col == 0) out[dv] = most, out[dv + 1] = l;
    }
  }
}

template <typename T, int GK, int GV>
__global__ void __launch_bounds__(64 * kStepWaves, kAtOnce<T>) softmax_step_packed_kernel(SoftmaxStepArgs a, SoftmaxStepPlan p) {
  extern __shared__ float sums_of[];  // [wave][member][dv]
  __shared__ StepState state[kStepWaves][kPackedMembers];
  __shared__ __attribute__((aligned(16))) uint8_t fresh[160];  // the new rows
  __shared__ __attribute__((aligned(16))) float scales[kStepWaves * 32 * (GK + 2 * GV)];
  StepPlace f;
  if (!find_stretch(a, p, f)) return;
  const int id = blockIdx.x, heads_of = a.H * p.blocks, head = f.hb / p.blocks;
  const int at = a.lengths[f.b], first = f.stretch * f.len * p.unit;
  const int64_t place = (int64_t)f.b * heads_of + f.hb;
  int2* const found = (int2*)a.scratch;
  float* const sums = (float*)(found + (int64_t)a.heads * p.blocks);
  if (p.bytes && f.stretch == 0 && threadIdx.x == 0) found[place] = int2{id, f.count};
  packed_stretch_rows<T, GK, GV>(a, (int64_t)f.b * a.H + head, f.hb - head * p.blocks, at, first,
                                 min(at + 1, first + f.len * p.unit),
                                 f.count == 1 ? nullptr : sums + (int64_t)id * min(kPackedMembers, a.G) * (a.dv_ + 2), sums_of,
                                 state, fresh, scales);
}

template <typename T, int GK, int GV>
hipError_t launch_step(const SoftmaxStepArgs& a, const SoftmaxStepPlan& p, hipStream_t s) {
  const int bytes = kStepWaves * std::min(kPackedMembers, a.G) * a.dv_ * (int)sizeof(float);  // (32 KB at most)
  hipLaunchKernelGGL((softmax_step_packed_kernel<T, GK, GV>), dim3(p.workgroups), dim3(64 * kStepWaves), bytes, s, a, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.bytes == 0) return e;
  hipLaunchKernelGGL((softmax_join_kernel<T, true>), dim3(a.heads * a.G), dim3((a.dv_ + 63) / 64 * 64), 0, s, a, p);
  return hipGetLastError();
}

template <typename T, int GK>
hipError_t launch_values(const SoftmaxStepArgs& a, const SoftmaxStepPlan& p, hipStream_t s) {
  switch (packed_groups(a.dv_)) {
    case 1: return launch_step<T, GK, 1>(a, p, s);
    case 2: return launch_step<T, GK, 2>(a, p, s);
    default: return launch_step<T, GK, 4>(a, p, s);
  }
}
template <typename T>
hipError_t launch_keys(const SoftmaxStepArgs& a, const SoftmaxStepPlan& p, hipStream_t s) {
  switch (packed_groups(a.dk_)) {
    case 1: return launch_values<T, 1>(a, p, s);
    case 2: return launch_values<T, 2>(a, p, s);
    default: return launch_values<T, 4>(a, p, s);
  }
}

}  // namespace

SoftmaxStepPlan plan_softmax_step_packed(bool bf16, int heads, int H, int G, int capacity, int dv) {
  return plan_softmax_step(bf16, heads, H, G, capacity, dv, kPackedMembers, 256 * (bf16 ? kAtOnce<uint16_t> : kAtOnce<float>));
}

hipError_t launch_softmax_step_packed(const SoftmaxStepArgs& a, bool bf16, hipStream_t s) {
  const SoftmaxStepPlan p = plan_softmax_step_packed(bf16, a.heads, a.H, a.G, a.capacity, a.dv_);
  return bf16 ? launch_keys<u16>(a, p, s) : launch_keys<float>(a, p, s);
}

}  // namespace sata
