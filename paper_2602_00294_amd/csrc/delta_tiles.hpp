// What the delta rule's kernels share: 16 x 16 products over 32 entries, and what a chunk's pairs leave for the scans.
//
// With G_i the sum of a chunk's log decays up to token i, S the state before the chunk and E the errors
// e_i - k_i S' of its tokens (u = beta E),
//     L_ij = exp(G_i - G_j) k_i.k_j (j < i),   E = (I + L beta)^-1 (v - exp(G) k S),
//     y    = c exp(G) q S + P E,  P_ij = c exp(G_i - G_j) q_i.k_j beta_j (j <= i),
//     S    = exp(G_C) S + sum_j exp(G_C - G_j) beta_j k_j (x) E_j,
// so that a chunk's tokens need one triangular inverse and products.  Differences of sums of logarithms are at
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

constexpr int kDeltaChunk = 32;
constexpr int kDeltaBlock = 64;  // tokens between the states that a gradient keeps

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

// eight values as an operand
template <int PL>
__device__ __forceinline__ void operand_of(float (&x)[8], uint4 (&op)[PL]) {
  uint4 w[1][PL];
  to_planes<PL>(x, w);
#pragma unroll
  for (int p = 0; p < PL; ++p) op[p] = w[0][p];
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

// What the pairs of a chunk leave, in the order in which lanes load it: operands [number][16 rows][lane].
template <bool BF16>
struct DeltaChunkData {
  static constexpr int kInverse = 3;            // numbers of an inverse's entry
  static constexpr int kPair = BF16 ? 2 : 3;    // of a pair's weight in the outputs
  uint4 inverse[kInverse][2][64];               // (I + L beta)^-1, rows i
  uint4 pairs[kPair][2][64];                    // P, rows i
  float early[32], late[32];                    // exp(G_i), beta_j exp(G_C - G_j)
  float whole[4];                               // exp(G_C)
};
// The same for gradients; `pairs` stays without use.
template <bool BF16>
struct DeltaChunkBack {
  uint4 inverse[3][2][64];  // (I + beta L)^-1 transposed, rows j
  uint4 pairs[3][2][64];    // c exp(G_i - G_j) q_i.k_j transposed, rows j
  float early[32], late[32], beta[32];  // exp(G_i), exp(G_C - G_j)
  float whole[4];
};

// The records of a head's chunks on their way into LDS.  (Loads have no branches: behind a branch the compiler waits for
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

// One column of a head's [rows][pitch] entries, a lane its own: entries of rows t0 + 16 x + 4 t4 .. +3 (x = 0, 1), zero behind
// the last row and where the lane has no column.  Stores there are dropped.
template <typename T>
struct ColumnStage {
  __amdgpu_buffer_rsrc_t rsrc;
  uint32_t off, pitch;
  int left;  // columns from this lane's on
  uint32_t r[8];
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
  template <int COUNT = 8>
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

hipError_t launch_delta_pairs(const DeltaArgs& a, bool bf16, void* data, void* back, hipStream_t s);
// The states before every block and the errors E of a call's tokens: what gradients start from.
hipError_t launch_delta_states(const DeltaArgs& a, bool bf16, const void* data, float* states, float* errors, hipStream_t s);
size_t delta_data_bytes(bool bf16, int heads, int n);

}  // namespace sata
