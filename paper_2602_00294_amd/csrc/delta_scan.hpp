// The gated delta rule's forward scan, for prompts (delta.hip) and for what gradients start from (delta_backward.hip).
//
// A wave has 16 columns of the state for a head's whole sequence, in the tiles of state_row; four of them share the staged
// queries and keys.  For a block (delta_tiles.hpp)
//     R = k S,  r = v - early R - (L_21 E_1 in the second half),  E = inverse r,
//     y = c early q S + P E,  S = whole S + k^T (late E),
// each a product whose right operand is what the one before left in this lane.  Four more waves bring the next block
// into LDS: issuing its loads costs a wave 3300 cycles of the 13000 that a block then took.
// 128 heads x 4096 tokens, d_k = d_v = 128, bfloat16: 255 us, 4 a block; matrix cores 37%, vector issue 40%, LDS 36% of
// the cycles, which one computing wave a SIMD overlaps only in part.  (16 columns are a product's least, and a head's
// states would have to be joined over waves if its rows were shared out: no second wave to a SIMD at 128 heads.)
//
// A few tokens cost what a block costs, and still less than one by one with a column of the state a thread: 32 heads of 128,
// pairs and scan, 13.7 us for 1 to 64 tokens, the other form 22.9 for one and 154 for 64.
#pragma once

#include <hip/hip_runtime.h>

#include "decay_power.hpp"
#include "delta_tiles.hpp"
#include "device_common.hpp"
#include "kernels.hpp"
#include "pair_tiles.hpp"

namespace sata {

constexpr int kScanWaves = 4, kScanThreads = 2 * 64 * kScanWaves;

// One of the buffers in LDS: a block's keys, queries, what its pairs left, and values of the workgroup's columns.
template <typename T, int ND>
struct DeltaLds {
  using L = DeltaTile<T, ND, kDeltaBlock>;
  using Data = DeltaForward<sizeof(T) == 2>;
  using V = SliceStage<T, 64 * kScanWaves>;
  static constexpr int kBuffers = sizeof(T) == 2 ? 2 : 1;
  static constexpr int kBuffer = 2 * L::kBytes + (int)sizeof(Data) + V::kBytes;
  static constexpr int kBytes = kBuffers * kBuffer;
  static_assert(kBytes <= 160 * 1024 && kBuffer % 16 == 0, "LDS of one workgroup");
};

// A block's tokens one by one, for blocks in which something is not finite: products would take it to earlier tokens,
// whose weights of it are zero.
template <typename T, int ND>
__device__ __forceinline__ void delta_one_by_one(const DeltaArgs& a, int head, int64_t shared, int t0, int m, int col, bool on,
                                                 f32x4 (&S)[2 * ND], T* y, float* errors) {
  const int t4 = (threadIdx.x & 63) >> 4;
  const T* const q = (const T*)a.q + shared * a.n * a.dk;
  const T* const k = (const T*)a.k + shared * a.n * a.dk;
  for (int t = t0; t < t0 + m; ++t) {
    const FloatPair lam = float_pair(exp(delta_rate(a.g[(int64_t)head * a.n + t])));
    const float beta = a.beta[(int64_t)head * a.n + t];
    float p = 0.f;
#pragma unroll 1
    for (int j = 0; j < 2 * ND; ++j) {
      f32x4 s = S[0];
#pragma unroll
      for (int x = 1; x < 2 * ND; ++x) s = j == x ? S[x] : s;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = state_row(j, i, t4);
        s[i] = times(s[i], lam);
        p = row < a.dk ? fmaf(entry_of(k, (int64_t)t * a.dk + row), s[i], p) : p;
      }
#pragma unroll
      for (int x = 0; x < 2 * ND; ++x) S[x] = j == x ? s : S[x];
    }
    p += __shfl_xor(p, 16);
    p += __shfl_xor(p, 32);
    const float e = on ? entry_of((const T*)a.v, ((int64_t)head * a.n + t) * a.dv + col) - p : 0.f;
    const float u = on ? beta * e : 0.f;
    if (errors && on && t4 == 0) errors[((int64_t)head * a.n + t) * a.dv + col] = e;
    p = 0.f;
#pragma unroll 1
    for (int j = 0; j < 2 * ND; ++j) {
      f32x4 s = S[0];
#pragma unroll
      for (int x = 1; x < 2 * ND; ++x) s = j == x ? S[x] : s;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = state_row(j, i, t4);
        s[i] = row < a.dk ? fmaf(entry_of(k, (int64_t)t * a.dk + row), u, s[i]) : s[i];
        p = row < a.dk ? fmaf(entry_of(q, (int64_t)t * a.dk + row), s[i], p) : p;
      }
#pragma unroll
      for (int x = 0; x < 2 * ND; ++x) S[x] = j == x ? s : S[x];
    }
    p += __shfl_xor(p, 16);
    p += __shfl_xor(p, 32);
    if (y && on && t4 == 0) y[(int64_t)t * a.dv + col] = rounded<T>(p * a.scale);
  }
}

// GRAD: no outputs, but the errors and the states before every block.
template <typename T, int ND, bool GRAD>
__device__ __forceinline__ void delta_scan(const DeltaArgs& a, const void* data_, float* states, float* errors, int workgroup,
                                           int slices, u16* smem16) {
  constexpr bool BF16 = sizeof(T) == 2;
  constexpr int C = kDeltaBlock, kHalf = 64 * kScanWaves;
  using D = DeltaLds<T, ND>;
  using L = typename D::L;
  using Data = typename D::Data;
  using V = typename D::V;
  constexpr int PE = Data::kPair, PY = BF16 ? 2 : 3;  // numbers of an error and of a state's entry in the outputs
  int head, slice;
  if (!delta_place(workgroup, a.heads, slices, head, slice)) return;
  const int tid = threadIdx.x, lane = tid & 63, l15 = lane & 15, t4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t shared = head / a.G;
  const int len = tokens_of(a.lengths, head / (a.Hk * a.G), a.n), blocks = (len + C - 1) / C;
  const int64_t all_blocks = (a.n + C - 1) / C;
  auto buffer = [&](int c) { return smem16 + (D::kBuffers == 2 && (c & 1) ? D::kBuffer / 2 : 0); };
  if (wave >= kScanWaves) {  // ---- the next block into LDS
    const int id = tid - kHalf;
    DeltaStage<T, ND, C, kHalf> sq, sk;
    DataStage<Data, kHalf> sd;
    V sv;
    sq.init((const T*)a.q + shared * a.n * a.dk, len, a.dk, id);
    sk.init((const T*)a.k + shared * a.n * a.dk, len, a.dk, id);
    sd.init((const Data*)data_ + head * all_blocks, blocks, id);
    sv.init((const T*)a.v + (int64_t)head * a.n * a.dv, len, a.dv, 64 * slice, id);
    auto fetch = [&](int c) {
      sk.fetch(c * C);
      if (!GRAD) sq.fetch(c * C);
      sd.fetch(c);
      sv.fetch(c * C);
    };
    if (blocks > 0) fetch(0);
    for (int c = 0; c < blocks; ++c) {
      u16* const tk = buffer(c);
      if (D::kBuffers == 1 && c > 0) __syncthreads();  // (the block before has been read)
      sk.put(tk, c * C);
      if (!GRAD) sq.put(tk + L::kElems, c * C);
      sd.put((Data*)(tk + 2 * L::kElems));
      sv.put((T*)((Data*)(tk + 2 * L::kElems) + 1), c * C);
      __syncthreads();
      if (c + 1 < blocks) fetch(c + 1);
    }
    return;
  }
  const int c0 = 16 * (kScanWaves * slice + wave), col = c0 + l15;
  const bool on = col < a.dv;
  const int64_t size = (int64_t)a.dk * a.dv;
  f32x4 S[2 * ND];
#pragma unroll
  for (int j = 0; j < 2 * ND; ++j) S[j] = zero4();
  StateColumns state;
  if (a.S_in) {
    state.init(a.S_in + head * size, a.dk, a.dv, col);
    state.load(S);
  }
  T* const y = GRAD ? nullptr : (T*)a.y + (int64_t)head * a.n * a.dv;
  const bool vec = a.dv % 4 == 0 && ((uintptr_t)y & (4 * sizeof(T) - 1)) == 0;
  {
    ColumnStage<float> se;
    if (GRAD) se.init(errors + (int64_t)head * a.n * a.dv, len, a.dv, col);
    for (int c = 0; c < blocks; ++c) {
      const int t0 = c * C;
      const u16* const tk = buffer(c);
      const u16* const tq = tk + L::kElems;
      const Data& d = *(const Data*)(tq + L::kElems);
      if (D::kBuffers == 1 && c > 0) __syncthreads();
      __syncthreads();
      const T* const v = (const T*)(&d + 1) + 16 * wave + l15;
      float r[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) r[e] = entry_of(v, (16 * (e >> 2) + 4 * t4 + (e & 3)) * V::kPitch);
      if (GRAD) {
        state.init(states + (head * all_blocks + c) * size, a.dk, a.dv, col);
        state.store(S);
      }
      // Operands are loaded well ahead of their products: with one wave a SIMD nothing else hides LDS's latency.
      f32x4 early[4], late[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        early[x] = *(const f32x4*)(d.early + 16 * x + 4 * t4);
        late[x] = *(const f32x4*)(d.late + 16 * x + 4 * t4);
      }
      const FloatPair whole = d.whole;
      auto operand = [&](const DeltaOperand* p, int x, auto& op) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(op) / sizeof(op[0])); ++i) op[i] = p[i][x][lane];
      };
      uint4 st[ND][3];
#pragma unroll
      for (int b = 0; b < ND; ++b) operand_of<3>(S[2 * b], S[2 * b + 1], st[b]);
      f32x4 R[4], o[4], E[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) R[x] = o[x] = zero4();
#pragma unroll
      for (int b = 0; b < ND; ++b) {
        uint4 e[4][L::kPl];
#pragma unroll
        for (int x = 0; x < 4; ++x) rows16<L>(tk, 16 * x, b, e[x]);
        dots_left16(e, st[b], R);
      }
      float bad = 0.f;  // (an infinity or NaN times zero is NaN)
      uint4 ep[2][3];
      auto errors_of = [&](int h, const f32x4 (&before)[2]) {
        uint4 inv[2][3];
#pragma unroll
        for (int x = 0; x < 2; ++x) operand(d.inverse[h], x, inv[x]);
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          z[e] = fmaf(-early[2 * h + (e >> 2)][e & 3], R[2 * h + (e >> 2)][e & 3], r[8 * h + e]) - before[e >> 2][e & 3];
          bad = fmaf(z[e], 0.f, bad);
        }
        uint4 rp[3];
        operand_of<3>(z, rp);
        f32x4 w[2] = {zero4(), zero4()};
        dots_left16(inv, rp, w);
        E[2 * h] = w[0], E[2 * h + 1] = w[1];
      };
      f32x4 before[2] = {zero4(), zero4()};
      errors_of(0, before);
      if constexpr (!GRAD) {  // (between the products that wait for each other)
#pragma unroll
        for (int b = 0; b < ND; ++b) {
          uint4 so[PY], e[4][L::kPl];
#pragma unroll
          for (int p = 0; p < PY; ++p) so[p] = st[b][p];
#pragma unroll
          for (int x = 0; x < 4; ++x) rows16<L>(tq, 16 * x, b, e[x]);
          dots_right16(so, e, o);
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) bad = fmaf(E[e >> 2][e & 3], 0.f, bad);
      operand_of<3>(E[0], E[1], ep[0]);
      {
        uint4 below[2][3];
#pragma unroll
        for (int x = 0; x < 2; ++x) operand(d.below, x, below[x]);
        dots_left16(below, ep[0], before);
      }
      auto add_pairs = [&](int h, int which, int x0) {  // of errors of half h to tokens 16 x0 .. +31
        uint4 pairs[2][PE], e[PE];
#pragma unroll
        for (int x = 0; x < 2; ++x) operand(d.pairs[which], x, pairs[x]);
#pragma unroll
        for (int p = 0; p < PE; ++p) e[p] = ep[h][p];
        f32x4 w[2] = {o[x0], o[x0 + 1]};
        dots_right16<PE - 1>(e, pairs, w);
        o[x0] = w[0], o[x0 + 1] = w[1];
      };
      if constexpr (!GRAD) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float readout = d.early[16 * x + l15] * a.scale;
#pragma unroll
          for (int i = 0; i < 4; ++i) o[x][i] *= readout;
        }
        add_pairs(0, 0, 0);
        add_pairs(0, 1, 2);
      }
      errors_of(1, before);
#pragma unroll
      for (int e = 8; e < 16; ++e) bad = fmaf(E[e >> 2][e & 3], 0.f, bad);
      settle_mfma();
      if (__builtin_expect(__ballot(!(bad == 0.f)) != 0, 0)) {
        delta_one_by_one<T, ND>(a, head, shared, t0, min(C, len - t0), col, on, S, y, GRAD ? errors : nullptr);
        continue;
      }
      uint4 wp[2][3];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = E[2 * h + (e >> 2)][e & 3] * late[2 * h + (e >> 2)][e & 3];
        operand_of<3>(w, wp[h]);
      }
      if (GRAD) {
#pragma unroll
        for (int e = 0; e < 16; ++e) se.store(t0, e, E[e >> 2][e & 3]);
      } else {
        operand_of<PE>(E[2], E[3], reinterpret_cast<uint4(&)[PE]>(ep[1]));
        add_pairs(1, 2, 2);
      }
#pragma unroll
      for (int j = 0; j < 2 * ND; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) S[j][i] = times(S[j][i], whole);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint4 e[2 * ND][L::kPl];
#pragma unroll
        for (int j = 0; j < 2 * ND; ++j) state_columns16<L>(tk, 32 * h, j, e[j]);
        dots_left16(e, wp[h], S);
      }
      if (!GRAD) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int t = t0 + 16 * x + l15;
          const float z[4] = {o[x][0], o[x][1], o[x][2], o[x][3]};
          if (t < len) store4<T>(y + (int64_t)t * a.dv, c0 + 4 * t4, a.dv, z, vec);
        }
      }
      settle_mfma();
    }
  }
  if (!GRAD && a.S_out) {
    state.init(a.S_out + head * size, a.dk, a.dv, col);
    state.store(S);
  }
  if (!GRAD && on) {  // rows behind the sequence
    for (int t = len + t4; t < a.n; t += 4) y[(int64_t)t * a.dv + col] = (T)0;
  }
}

}  // namespace sata
