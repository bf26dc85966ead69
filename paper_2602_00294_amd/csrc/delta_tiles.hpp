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

// Rows in LDS as PairTile has them, with the 16-byte units of a row in places of their own: here 32 lanes read 16 rows of
// one unit or, transposed, 8 rows of two neighbouring ones, and each meets every bank once.
template <typename T, int ND, int ROWS>
struct DeltaTile : PairTile<T, ND, ROWS> {
  using P = PairTile<T, ND, ROWS>;
  __device__ static __forceinline__ int swap(int row) {
    if constexpr (P::kUnits == 16) return ((row & 7) << 1) | ((row >> 3) & 1);
    else if constexpr (P::kUnits == 8) return (((row >> 1) & 3) << 1) | ((row >> 3) & 1);
    else return (((row >> 2) & 1) << 1) | ((row >> 3) & 1);
  }
  __device__ static __forceinline__ int at(int row, int col) { return row * P::kRow + 8 * ((col >> 3) ^ swap(row)) + (col & 7); }
};
template <typename T, int ND, int ROWS, int THREADS>
using DeltaStage = TileStage<T, ND, ROWS, THREADS, DeltaTile<T, ND, ROWS>>;

// Sums of the products a[i] b[j] with i + j <= MAX, smallest first, for N results at once, product by product: a result's own
// products wait for each other.
template <int MAX = 2, int N, int NA, int NB>
__device__ __forceinline__ void dots_left16(const uint4 (&a)[N][NA], const uint4 (&b)[NB], f32x4 (&c)[N]) {
#pragma unroll
  for (int t = MAX; t >= 0; --t)
#pragma unroll
    for (int i = 0; i <= t; ++i)
      if (i < NA && t - i < NB)
#pragma unroll
        for (int x = 0; x < N; ++x) c[x] = mfma_bf16(a[x][i], b[t - i], c[x]);
}
template <int MAX = 2, int N, int NA, int NB>
__device__ __forceinline__ void dots_right16(const uint4 (&a)[NA], const uint4 (&b)[N][NB], f32x4 (&c)[N]) {
#pragma unroll
  for (int t = MAX; t >= 0; --t)
#pragma unroll
    for (int i = 0; i <= t; ++i)
      if (i < NA && t - i < NB)
#pragma unroll
        for (int x = 0; x < N; ++x) c[x] = mfma_bf16(a[i], b[x][t - i], c[x]);
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

// Operands out of a tile of rows (L: DeltaTile).
// Rows r0 .. +15, entries 32 s .. +31: lane t4 has entries 32 s + 8 t4 .. +7.
template <typename L>
__device__ __forceinline__ void rows16(const u16* t, int r0, int s, uint4 (&op)[L::kPl]) {
  const int lane = threadIdx.x & 63, row = r0 + (lane & 15), t4 = lane >> 4;
  const u16* const p = t + row * L::kRow + 8 * ((4 * s + t4) ^ L::swap(row));
#pragma unroll
  for (int i = 0; i < L::kPl; ++i) op[i] = *(const uint4*)(p + i * L::kPlane);
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
// The scans' states have rows of their own order: row r of tile 2 b + x is entry 32 b + 8 (r / 4) + 4 x + r % 4 of a key, so that
// two tiles' numbers contract with a key's entries in the order in which rows16 reads them.
__device__ __forceinline__ int state_row(int j, int i, int t4) { return 32 * (j >> 1) + 8 * t4 + 4 * (j & 1) + i; }
// The entries of tile j over rows r0 .. +31 in the order of a result's rows.
template <typename L>
__device__ __forceinline__ void state_columns16(const u16* t, int r0, int j, uint4 (&op)[L::kPl]) {
  const int lane = threadIdx.x & 63, l15 = lane & 15, t4 = lane >> 4;
  const int row = r0 + 4 * t4 + (l15 >> 2), unit = 4 * (j >> 1) + (l15 & 3), half = 4 * (j & 1);
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
  FloatPair whole;                            // exp(G_C), of which a state takes one for every block
  float none[2];
};
// For gradients, transposed: beta belongs to the other side there, M_ij = exp(G_i - G_j) beta_i k_i.k_j.
struct DeltaBackward {
  DeltaOperand inverse[2][3];  // (I + M_11)^-T, (I + M_22)^-T, rows j
  DeltaOperand below[3];       // M_21^T, rows j
  DeltaOperand pairs[3][3];    // P_11^T, P_21^T, P_22^T without beta, rows j
  float early[kDeltaBlock], late[kDeltaBlock], beta[kDeltaBlock];  // exp(G_i), exp(G_C - G_j)
  FloatPair whole;
  float none[2];
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

// A lane's own column of a head's [rows][width] entries: entries of rows t0 + 16 x + 4 t4 .. +3 (x = 0 .. 3) are written, those behind
// the last row and of a lane without a column dropped.
template <typename T>
struct ColumnStage {
  __amdgpu_buffer_rsrc_t rsrc;
  uint32_t off, pitch;
  __device__ __forceinline__ void init(const T* head, int rows, int width, int col) {
    rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(head), 0, rows * width * (int)sizeof(T), 0x00020000);
    pitch = (uint32_t)(width * (int)sizeof(T));
    off = col < width ? (uint32_t)((threadIdx.x & 63) >> 4) * 4u * pitch + (uint32_t)(col * (int)sizeof(T)) : kNoVector;
  }
  __device__ __forceinline__ int at(int t0, int e) const { return (int)(off + (uint32_t)(t0 + 16 * (e >> 2) + (e & 3)) * pitch); }
  __device__ __forceinline__ void store(int t0, int e, float x) const {
    if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x), rsrc, at(t0, e), 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b16((unsigned short)(pack2(x, 0.f) & 0xffffu), rsrc, at(t0, e), 0, 0);
  }
};

// Eight entries c0 .. +7 of a row of a head's [rows][width]: by vectors where the rows allow them.  Rows behind the last and
// columns behind the width read as zero and are not written.  (No branch but the one on `vec`, the same for all.)
template <typename T>
struct RowAccess {
  __amdgpu_buffer_rsrc_t rsrc;
  int width;
  bool vec;
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  __device__ __forceinline__ void init(const T* head, int rows, int width_) {
    width = width_;
    vec = width * (int)sizeof(T) % 16 == 0 && ((uintptr_t)head & 15) == 0;
    rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(head), 0, rows * width * (int)sizeof(T), 0x00020000);
  }
  __device__ __forceinline__ int at(int row, int col) const {
    return (int)(col < width ? (uint32_t)(row * width + col) * (uint32_t)sizeof(T) : kNoVector);
  }
  __device__ __forceinline__ uint4 quad(int offset) const {
    return __builtin_bit_cast(uint4, (u32x4)__builtin_amdgcn_raw_buffer_load_b128(rsrc, offset, 0, 0));
  }
  // (float32 rows alone are read here: blocks of bfloat16 ones go through LDS)
  __device__ __forceinline__ void load(int row, int c0, float (&x)[8]) const {
    static_assert(sizeof(T) == 4, "float32 rows");
    if (vec) {
      const uint4 w = quad(at(row, c0)), v = quad(at(row, c0 + 4));
      x[0] = __uint_as_float(w.x), x[1] = __uint_as_float(w.y), x[2] = __uint_as_float(w.z), x[3] = __uint_as_float(w.w);
      x[4] = __uint_as_float(v.x), x[5] = __uint_as_float(v.y), x[6] = __uint_as_float(v.z), x[7] = __uint_as_float(v.w);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __uint_as_float((uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rsrc, at(row, c0 + i), 0, 0));
    }
  }
  template <int PL>
  __device__ __forceinline__ void operand(int row, int c0, uint4 (&op)[PL]) const {
    float x[8];
    load(row, c0, x);
    operand_of<PL>(x, op);
  }
  __device__ __forceinline__ void put_quad(int offset, uint32_t a, uint32_t b, uint32_t c, uint32_t d) const {
    __builtin_amdgcn_raw_buffer_store_b128(u32x4{a, b, c, d}, rsrc, offset, 0, 0);
  }
  __device__ __forceinline__ void store(int row, int c0, const float (&x)[8]) const {
    if (vec) {
      if constexpr (sizeof(T) == 2) {
        put_quad(at(row, c0), pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
      } else {
#pragma unroll
        for (int h = 0; h < 8; h += 4)
          put_quad(at(row, c0 + h), __float_as_uint(x[h]), __float_as_uint(x[h + 1]), __float_as_uint(x[h + 2]), __float_as_uint(x[h + 3]));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16((unsigned short)(pack2(x[i], 0.f) & 0xffffu), rsrc, at(row, c0 + i), 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x[i]), rsrc, at(row, c0 + i), 0, 0);
      }
    }
  }
};

// 64 rows of a slice of 64 columns of a head's [rows][width] entries on their way into LDS, as they are.
template <typename T, int THREADS>
struct SliceStage {
  static constexpr int kPitch = 68;  // entries of a row in LDS: the four rows that a wave reads at once lie in other banks
  static constexpr int kBytes = kDeltaBlock * kPitch * (int)sizeof(T);
  static constexpr int kEV = 16 / (int)sizeof(T), kUnits = 64 / kEV, kIt = kDeltaBlock * kUnits / THREADS;
  const T* base;
  VectorReader read;
  int rows, width, c0, tid;
  bool vec;
  uint32_t off, pitch;
  uint4 r[kIt];
  __device__ __forceinline__ void init(const T* head, int rows_, int width_, int c0_, int tid_) {
    base = head, rows = rows_, width = width_, c0 = c0_, tid = tid_;
    vec = width % kEV == 0 && ((uintptr_t)head & 15) == 0;
    read = VectorReader(head, vec ? (int64_t)rows * width * (int)sizeof(T) : 0);
    pitch = (uint32_t)(width * (int)sizeof(T));
    const int col = c0 + tid % kUnits * kEV;
    off = col < width ? (uint32_t)(tid / kUnits) * pitch + (uint32_t)(col * (int)sizeof(T)) : kNoVector;
  }
  __device__ __forceinline__ void fetch(int t0) {
#pragma unroll
    for (int i = 0; i < kIt; ++i) r[i] = read(off + (uint32_t)(t0 + i * (THREADS / kUnits)) * pitch);
  }
  __device__ __forceinline__ void put(T* t, int t0) const {
    if (vec) {
#pragma unroll
      for (int i = 0; i < kIt; ++i) {
        T* const p = t + (tid / kUnits + i * (THREADS / kUnits)) * kPitch + tid % kUnits * kEV;
        *(uint2*)p = uint2{r[i].x, r[i].y};
        *(uint2*)(p + kEV / 2) = uint2{r[i].z, r[i].w};
      }
    } else {
      for (int i = tid; i < kDeltaBlock * 64; i += THREADS) {
        const int row = i / 64, col = i % 64;
        t[row * kPitch + col] = t0 + row < rows && c0 + col < width ? base[(int64_t)(t0 + row) * width + c0 + col] : (T)0;
      }
    }
  }
};

// A state of [dk][dv] entries, its tiles j of a wave's 16 columns from memory and back.
struct StateColumns {
  __amdgpu_buffer_rsrc_t rsrc;
  uint32_t off, pitch;
  __device__ __forceinline__ void init(const float* state, int dk, int dv, int col) {
    rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(state), 0, dk * dv * 4, 0x00020000);
    pitch = (uint32_t)dv * 4u;
    off = col < dv ? (uint32_t)col * 4u : kNoVector;
  }
  __device__ __forceinline__ int at(int j, int i) const {
    return (int)(off + (uint32_t)state_row(j, i, (threadIdx.x & 63) >> 4) * pitch);
  }
  template <int N>
  __device__ __forceinline__ void load(f32x4 (&S)[N]) const {
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) S[j][i] = __uint_as_float((uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rsrc, at(j, i), 0, 0));
  }
  template <int N>
  __device__ __forceinline__ void store(const f32x4 (&S)[N]) const {
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(S[j][i]), rsrc, at(j, i), 0, 0);
  }
};

// Workgroups to heads and slices of columns: an XCD takes whole heads, whose queries and keys are then read through one L2.
__device__ __forceinline__ bool delta_place(int workgroup, int heads, int slices, int& head, int& slice) {
  if (heads >= 8) {
    const int j = workgroup >> 3;
    head = j / slices * 8 + (workgroup & 7);
    slice = j % slices;
    return head < heads;
  }
  head = workgroup / slices;
  slice = workgroup % slices;
  return true;
}
inline unsigned delta_grid(int heads, int slices) { return (unsigned)((heads >= 8 ? (heads + 7) / 8 * 8 : heads) * slices); }

// Records [head][block] of DeltaForward and, where `backward`, DeltaBackward.
hipError_t launch_delta_pairs(const DeltaArgs& a, bool bf16, void* forward, void* backward, hipStream_t s);
size_t delta_forward_bytes(bool bf16, int heads, int n);

}  // namespace sata
