// What the delta rule's kernels share: 16 x 16 products over 32 entries, and what the pairs of a block's tokens leave for
// the scans.
//
// A block is 64 tokens, two halves of 32.  With G_i the sum of its log decays up to token i, S the state before it and
// E_i = v_i - k_i S' the errors of its tokens (u = beta E),
//     L_ij = exp(G_i - G_j) beta_j k_i.k_j (j < i),   E = (I + L)^-1 (v - exp(G) k S): half by half,
//     E_1  = (I + L_11)^-1 (v_1 - exp(G) k_1 S),      E_2 = (I + L_22)^-1 (v_2 - exp(G) k_2 S - L_21 E_1),
//     y    = c exp(G) q S + P E,  P_ij = c exp(G_i - G_j) beta_j q_i.k_j (j <= i),
//     S    = exp(G_C) S + sum_j exp(G_C - G_j) beta_j k_j (x) E_j,
// so that a block's tokens need triangular inverses of 32 x 32 and products.  Differences of sums of logarithms are at
// most 0: no factor overflows, however strong the decay.
//
// Products are v_mfma_f32_16x16x32_bf16.  Lane l (l15 = l % 16, t4 = l / 16) holds row (left operand) or column
// (right) l15 and entries 8 t4 .. +7 of the contraction, and of a result column l15, rows 4 t4 .. +3.  So the
// numbers of two results, rows 0..15 and 16..31, are an operand that contracts over these 32 rows in the
// order {4 t4 .. +3, 16 + 4 t4 .. +3}, lane by lane: states, errors and pairs stay in their lanes.
#pragma once

#include <hip/hip_runtime.h>

#include "decay_power.hpp"
#include "device_common.hpp"
#include "kernels.hpp"
#include "pair_tiles.hpp"

namespace sata {

constexpr int kDeltaBlock = 64;

__device__ __forceinline__ f32x4 zero4() { return f32x4{0.f, 0.f, 0.f, 0.f}; }

// sum of the products a[i] b[j] with i + j <= MAX, smallest first
template <int MAX = 2, int NA, int NB>
__device__ __forceinline__ f32x4 dot_planes16(const uint4 (&a)[NA], const uint4 (&b)[NB], f32x4 c) {
#pragma unroll
  for (int t = MAX; t >= 0; --t)
#pragma unroll
    for (int i = 0; i <= t; ++i)
      if (i < NA && t - i < NB) c = mfma_bf16(a[i], b[t - i], c);
  return c;
}

// Eight values as an operand of PL bfloat16 numbers each; x becomes what they leave out.  What two numbers leave out is
// one v_dot2_f32_bf16 each, x - (first, 0) or - (0, second): exact, and it takes the place of unpacking and subtracting.
// (An infinity makes NaN of its neighbour too.  The factors lie in registers: as an inline constant the first
// would be multiplied with both numbers.)
template <int PL>
__device__ __forceinline__ void operand_of(float (&x)[8], uint4 (&op)[PL]) {
  uint32_t first = 0x0000bf80u, second = 0xbf800000u;
  asm("" : "+s"(first), "+s"(second));
  typedef __bf16 pair __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int p = 0; p < PL; ++p) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = pack2(x[2 * i], x[2 * i + 1]);
      if (p + 1 < PL) {
        const pair v = __builtin_bit_cast(pair, w[i]);
        x[2 * i] = __builtin_amdgcn_fdot2_f32_bf16(v, __builtin_bit_cast(pair, first), x[2 * i], false);
        x[2 * i + 1] = __builtin_amdgcn_fdot2_f32_bf16(v, __builtin_bit_cast(pair, second), x[2 * i + 1], false);
      }
    }
    op[p] = uint4{w[0], w[1], w[2], w[3]};
  }
}
template <int PL>
__device__ __forceinline__ void operand_of(const f32x4& a, const f32x4& b, uint4 (&op)[PL]) {
  float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  operand_of<PL>(x, op);
}

// Operands out of a tile of rows (L: PairTile).
// Rows r0 .. +15, entries 32 s .. +31 in their order.
template <typename L>
__device__ __forceinline__ void rows16(const u16* t, int r0, int s, uint4 (&op)[L::kPl]) {
  const int lane = threadIdx.x & 63, row = r0 + (lane & 15), t4 = lane >> 4;
  const u16* const p = t + row * L::kRow + 8 * ((4 * s + t4) ^ L::swap(row));
#pragma unroll
  for (int i = 0; i < L::kPl; ++i) op[i] = *(const uint4*)(p + i * L::kPlane);
}
// The same in the order of a result's rows.
template <typename L>
__device__ __forceinline__ void rows16_as_results(const u16* t, int r0, int s, uint4 (&op)[L::kPl]) {
  const int lane = threadIdx.x & 63, row = r0 + (lane & 15), t4 = lane >> 4;
  const u16* const p = t + row * L::kRow + 4 * (t4 & 1);
  const u16* const a = p + 8 * ((4 * s + (t4 >> 1)) ^ L::swap(row));
  const u16* const b = p + 8 * ((4 * s + 2 + (t4 >> 1)) ^ L::swap(row));
#pragma unroll
  for (int i = 0; i < L::kPl; ++i) {
    const uint2 x = *(const uint2*)(a + i * L::kPlane), y = *(const uint2*)(b + i * L::kPlane);
    op[i] = uint4{x.x, x.y, y.x, y.y};
  }
}
// Columns 16 j .. +15 over rows r0 .. +31 in the order of a result's rows.
template <typename L>
__device__ __forceinline__ void columns16(const u16* t, int r0, int j, uint4 (&op)[L::kPl]) {
  const int lane = threadIdx.x & 63, l15 = lane & 15, t4 = lane >> 4;
  const int row = r0 + 4 * t4 + (l15 >> 2), unit = 2 * j + ((l15 & 3) >> 1), half = 4 * (l15 & 1);
  const u16* const a = t + row * L::kRow + 8 * (unit ^ L::swap(row)) + half;
  const u16* const b = t + (row + 16) * L::kRow + 8 * (unit ^ L::swap(row + 16)) + half;
#pragma unroll
  for (int i = 0; i < L::kPl; ++i) op[i] = read_transposed(a + i * L::kPlane, (int)(b - a));
}

// What the pairs of a block leave, in the order in which lanes load it: operands [number][16 rows][lane] of 32 rows.
typedef uint4 DeltaOperand[2][64];
template <bool BF16>
struct DeltaForward {
  static constexpr int kPair = BF16 ? 2 : 3;  // numbers of a pair's weight in the outputs
  DeltaOperand inverse[2][3];                 // (I + L_11)^-1, (I + L_22)^-1, rows i
  DeltaOperand below[3];                      // L_21, rows i
  DeltaOperand pairs[3][kPair];               // P_11, P_21, P_22, rows i
  float early[kDeltaBlock], late[kDeltaBlock];  // exp(G_i), beta_j exp(G_C - G_j)
  float whole[4];                             // exp(G_C)
};
// For gradients, transposed: beta belongs to the other side there, M_ij = exp(G_i - G_j) beta_i k_i.k_j.
struct DeltaBackward {
  DeltaOperand inverse[2][3];  // (I + M_11)^-T, (I + M_22)^-T, rows j
  DeltaOperand below[3];       // M_21^T, rows j
  DeltaOperand pairs[3][3];    // P_11^T, P_21^T, P_22^T without beta, rows j
  float early[kDeltaBlock], late[kDeltaBlock], beta[kDeltaBlock];  // exp(G_i), exp(G_C - G_j)
  float whole[4];
};

// The records of a head's blocks on their way into LDS.  (Loads have no branches: behind a branch the compiler waits for
// all that are on their way.)
template <typename D, int THREADS>
struct DataStage {
  static_assert(sizeof(D) % 16 == 0, "whole vectors");
  static constexpr int kVectors = sizeof(D) / 16, kIt = (kVectors + THREADS - 1) / THREADS;
  VectorReader read;
  int tid;
  uint4 r[kIt];
  __device__ __forceinline__ void init(const D* records, int count, int tid_) {
    read = VectorReader(records, (int64_t)count * sizeof(D));
    tid = tid_;
  }
  __device__ __forceinline__ void fetch(int c) {
#pragma unroll
    for (int i = 0; i < kIt; ++i) r[i] = read((uint32_t)c * (uint32_t)sizeof(D) + 16u * (uint32_t)(tid + i * THREADS));
  }
  __device__ __forceinline__ void put(D* d) const {
#pragma unroll
    for (int i = 0; i < kIt; ++i)
      if ((i + 1) * THREADS <= kVectors || tid + i * THREADS < kVectors) ((uint4*)d)[tid + i * THREADS] = r[i];
  }
};

// One column of a head's [rows][width] entries, a lane its own: entries of rows t0 + 16 x + 4 t4 .. +3 (x = 0 .. 3), zero behind
// the last row and where the lane has no column.  Stores there are dropped.
template <typename T>
struct ColumnStage {
  __amdgpu_buffer_rsrc_t rsrc;
  uint32_t off, pitch;
  int left;  // columns from this lane's on
  uint32_t r[16];
  __device__ __forceinline__ void init(const T* head, int rows, int width, int col) {
    rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(head), 0, rows * width * (int)sizeof(T), 0x00020000);
    pitch = (uint32_t)(width * (int)sizeof(T));
    left = width - col;
    off = (uint32_t)((threadIdx.x & 63) >> 4) * 4u * pitch + (uint32_t)(col * (int)sizeof(T));
  }
  // (of the column `ahead` further on, of which the lane may have none)
  __device__ __forceinline__ uint32_t at(int t0, int e, int ahead) const {
    const uint32_t place = off + (uint32_t)(t0 + 16 * (e >> 2) + (e & 3)) * pitch + (uint32_t)(ahead * (int)sizeof(T));
    return ahead < left ? place : kNoVector;
  }
  template <int COUNT = 16>
  __device__ __forceinline__ void fetch(int t0, int ahead = 0) {
#pragma unroll
    for (int e = 0; e < COUNT; ++e) {
      if constexpr (sizeof(T) == 4) r[e] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rsrc, (int)at(t0, e, ahead), 0, 0);
      else r[e] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rsrc, (int)at(t0, e, ahead), 0, 0);
    }
  }
  __device__ __forceinline__ float value(int e) const { return __uint_as_float(sizeof(T) == 4 ? r[e] : r[e] << 16); }
  __device__ __forceinline__ void store(int t0, int e, float x, int ahead = 0) const {
    if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x), rsrc, (int)at(t0, e, ahead), 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b16((unsigned short)(pack2(x, 0.f) & 0xffffu), rsrc, (int)at(t0, e, ahead), 0, 0);
  }
};

// Workgroups to heads and slices of columns: an XCD takes whole heads, whose queries and keys are then read through one L2.
__device__ __forceinline__ bool delta_place(int heads, int slices, int& head, int& slice) {
  if (heads >= 8) {
    const int j = blockIdx.x >> 3;
    head = j / slices * 8 + (int)(blockIdx.x & 7);
    slice = j % slices;
    return head < heads;
  }
  head = blockIdx.x / slices;
  slice = blockIdx.x % slices;
  return true;
}
inline unsigned delta_grid(int heads, int slices) { return (unsigned)((heads >= 8 ? (heads + 7) / 8 * 8 : heads) * slices); }

// Records [head][block] of DeltaForward and, where `backward`, DeltaBackward.
hipError_t launch_delta_pairs(const DeltaArgs& a, bool bf16, void* forward, void* backward, hipStream_t s);
size_t delta_forward_bytes(bool bf16, int heads, int n);
// The states before every block and the errors E of a call's tokens: what gradients start from.
hipError_t launch_delta_states(const DeltaArgs& a, bool bf16, const void* forward, float* states, float* errors, hipStream_t s);

}  // namespace sata
