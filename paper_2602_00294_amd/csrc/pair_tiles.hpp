// Tiles of rows in LDS and 32 x 32 matrix products of them, for the kernels of
// softmax attention and of linear attention with a decay.
//
// Products are v_mfma_f32_32x32x16_bf16.  Lane l (l31 = l % 32, h = l / 32) holds row
// (left operand) or column (right operand) l31 of a 32 x 16 operand, entries 8 h .. +7
// of the contraction, and column l31, rows 8 (i / 4) + 4 h + i % 4 of a result's 16
// numbers.  So numbers 0..7 and 8..15 of a result are, lane by lane, the right (or
// left) operands of a product that contracts over the result's rows 0..15 and
// 16..31, with the rows in the order {4 h .. +3, 8 + 4 h .. +3}: load_transposed reads
// the other operand in that order, and probabilities and states never leave their
// lanes.
//
// A tile holds rows of a tensor as they lie in memory, bfloat16, float32 ones as three
// bfloat16 numbers (planes) whose sum carries 24 bits; a product of two such numbers is
// the six partial products of order 2^-16 and up, accumulated in float32.  (Those beyond
// bfloat16's range, infinities among them: far_part.)  Rows are
// whole 64, 128 or 256 bytes; the 16-byte units of a row change places by
// its number, so that both ways of reading, along 16 or more rows and transposed by
// four rows of 64 bytes, meet every bank once.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "device_common.hpp"
#include "series.hpp"

namespace sata {

typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 mfma32(const uint4& a, const uint4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}
// sum of the products a[i] b[j] with i + j <= MAX, smallest first
template <int MAX = 2, int NA, int NB>
__device__ __forceinline__ f32x16 dot_planes32(const uint4 (&a)[NA], const uint4 (&b)[NB], f32x16 c) {
#pragma unroll
  for (int t = MAX; t >= 0; --t)
#pragma unroll
    for (int i = 0; i <= t; ++i)
      if (i < NA && t - i < NB) c = mfma32(a[i], b[t - i], c);
  return c;
}
__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}
// Idle cycles between a 32 x 32 matrix instruction and a branch behind which its
// results are read or overwritten (see settle_mfma for the compiler's distance
// across branches).
__device__ __forceinline__ void settle_mfma32() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15\n\ts_nop 3");
  __builtin_amdgcn_sched_barrier(0);
}
// Keeps what follows inside its branch: the compiler would rather compute both ways (the test of a tile
// for values that are not finite, 170 instructions, for every tile instead of one).
__device__ __forceinline__ void stay_in_branch() { asm volatile(""); }

__device__ __forceinline__ float entry_of(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float entry_of(const u16* p, int64_t i) { return __uint_as_float((uint32_t)p[i] << 16); }

// Row of a result's number i.
__device__ __forceinline__ int result_row(int i, int h) { return 8 * (i >> 2) + 4 * h + (i & 3); }

// Float32 values beyond bfloat16's largest number, 3.39e38, do not split as others do: rounded they would be
// infinite, and an infinity leaves NaN.  A finite one's first plane is that number; an infinity is (1, 0, infinity) with
// its sign, so that of the partial products with another value's planes one is infinite, the one with
// the other's first plane, whose sign and zero are the value's.  Tiles are looked over for such values behind their stores
// and put once more where there are some: 16 heads of 1000 tokens, d = 64, float32, prompts 41 -> 42 us and gradients
// 119 -> 121, of 2000 tokens 101 -> 108 and 288 -> 295; 32 heads of 2000, d = 128, 214 -> 217 and 826 -> 845; the same
// by the decay 151 -> 154 and 313 -> 324 (looked over before the stores: 220 and 855, 155 and 320).
// far_part: plane `plane` of what the planes before it left.
constexpr float kLargestBf16 = 0x1.fep127f;
__device__ __forceinline__ float far_part(float x, int plane) {
  if (plane == 2) return x;
  if (fabsf(x) == INFINITY) return plane == 0 ? copysignf(1.f, x) : 0.f;
  return fabsf(x) > kLargestBf16 ? copysignf(kLargestBf16, x) : x;
}

// N values (a multiple of 8) as operands of PL planes each; x is used up.  (For weights and states: an
// infinite one of several planes becomes NaN.)
template <int PL, int N>
__device__ __forceinline__ void to_planes(float (&x)[N], uint4 (&op)[N / 8][PL]) {
#pragma unroll
  for (int s = 0; s < N / 8; ++s)
#pragma unroll
    for (int p = 0; p < PL; ++p) {
      op[s][p] = to_bf16(x + 8 * s);
      if (p + 1 < PL) take_bf16(op[s][p], x + 8 * s);
    }
}

// ROWS rows of up to 32 ND columns of type T (u16: bfloat16 bits, or float).
template <typename T, int ND, int ROWS>
struct PairTile {
  static constexpr int kPl = sizeof(T) == 4 ? 3 : 1;
  static constexpr int kUnits = ND == 1 ? 4 : ND == 2 ? 8 : 16;  // 16-byte units in a row of a plane
  static constexpr int kRow = 8 * kUnits;                        // u16
  static constexpr int kPlane = ROWS * kRow;
  static constexpr int kElems = kPl * kPlane;
  static constexpr int kBytes = 2 * kElems;

  // Where a row's unit 0 is put; unit u is at u ^ swap(row).
  __device__ static __forceinline__ int swap(int row) {
    if constexpr (kUnits == 16) return ((row & 3) << 2) | ((row >> 2) & 3);
    else if constexpr (kUnits == 8) return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    else return (row >> 2) & 3;
  }
  __device__ static __forceinline__ int at(int row, int col) { return row * kRow + 8 * ((col >> 3) ^ swap(row)) + (col & 7); }

  // Operand of rows r0 .. r0 + 31 (r0 a multiple of 32), entries 16 s .. +15.
  __device__ static __forceinline__ void load_rows(const u16* t, int r0, int s, uint4 (&op)[kPl]) {
    const int lane = threadIdx.x & 63, l31 = lane & 31, h = lane >> 5;
    const u16* const p = t + (r0 + l31) * kRow + 8 * ((2 * s + h) ^ swap(l31));
#pragma unroll
    for (int i = 0; i < kPl; ++i) op[i] = *(const uint4*)(p + i * kPlane);
  }
  // Operand of columns 32 j .. +31 over the 16 rows from r0 (a multiple of 16).
  __device__ static __forceinline__ void load_transposed(const u16* t, int r0, int j, uint4 (&op)[kPl]) {
    const int lane = threadIdx.x & 63, l15 = lane & 15, g = (lane >> 4) & 1, h = lane >> 5;
    const int row = 4 * h + (l15 >> 2), unit = 4 * j + 2 * g + ((l15 & 3) >> 1), half = 4 * (l15 & 1);
    const u16* const a = t + (r0 + row) * kRow + 8 * (unit ^ swap(row)) + half;
    const u16* const b = t + (r0 + row + 8) * kRow + 8 * (unit ^ swap(row + 8)) + half;
#pragma unroll
    for (int i = 0; i < kPl; ++i) op[i] = read_transposed(a + i * kPlane, (int)(b - a));
  }
};

// The entries of a plane that are infinite or NaN, all bits of each set.  (A value's last plane is, where the value is.)
__device__ __forceinline__ uint4 not_finite_entries(const uint4& w) {
  auto wide = [](uint32_t x) { return ((((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u) >> 15) * 0xffffu; };
  return uint4{wide(w.x), wide(w.y), wide(w.z), wide(w.w)};
}

// 32 x 32 products of the tile's rows r0 .. +31 with this wave's rows.
template <typename L, int ND>
__device__ __forceinline__ f32x16 dot_rows32(const u16* t, int r0, const uint4 (&own)[2 * ND][L::kPl]) {
  f32x16 s = zero16();
#pragma unroll
  for (int i = 0; i < 2 * ND; ++i) {
    uint4 f[L::kPl];
    L::load_rows(t, r0, i, f);
    s = dot_planes32(f, own[i], s);
  }
  return s;
}

// acc[j] += (rows r0 .. r0 + 31 of the tile, columns 32 j .. +31)^T times the 32 x 32 weights w (of PW numbers each).
template <typename L, int ND, int PW>
__device__ __forceinline__ void contract32(const u16* t, int r0, const uint4 (&w)[2][PW], f32x16 (&acc)[ND]) {
#pragma unroll
  for (int j = 0; j < ND; ++j)
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      uint4 a[L::kPl];
      L::load_transposed(t, r0 + 16 * s, j, a);
      acc[j] = dot_planes32(a, w[s], acc[j]);
    }
}

// A tile on the diagonal has masked pairs, and a masked weight's zero times a value that is not
// finite would be no zero.  So such a tile (tile_not_finite) stays out of the
// products, and the wave goes over its rows one by one at the end with these two:
// this lane's column times a row, and acc += weight times a row.
template <typename T, int ND, int PL>
__device__ __forceinline__ float dot_row(const uint4 (&own)[2 * ND][PL], const T* row, int width) {
  const int h = (threadIdx.x & 63) >> 5;
  float r = 0.f;
#pragma unroll
  for (int s = 0; s < 2 * ND; ++s) {
    __builtin_amdgcn_sched_barrier(0);  // (a few entries at a time: registers)
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = PL - 1; i >= 0; --i) {
      uint32_t w[4] = {own[s][i].x, own[s][i].y, own[s][i].z, own[s][i].w};
      // (unpacked for each row anew: all of them, kept over the loop, would take the sweep's registers)
      asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]));
#pragma unroll
      for (int j = 0; j < 4; ++j) x[2 * j] += lo_f32(w[j]), x[2 * j + 1] += hi_f32(w[j]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int col = 16 * s + 8 * h + j;
      if (col < width) r = fmaf(x[j], entry_of(row, col), r);
    }
  }
  return r + __shfl_xor(r, 32);
}
template <typename T, int ND>
__device__ __forceinline__ void add_row(const T* row, int width, float weight, f32x16 (&acc)[ND]) {
  const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int j = 0; j < ND; ++j)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int col = 32 * j + result_row(i, h);
      if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
      if (col < width) acc[j][i] = fmaf(weight, entry_of(row, col), acc[j][i]);
    }
}

// Whether there are any (bits set).
__device__ __forceinline__ uint32_t not_finite_bits(const uint4& w) {
  return ((((w.x & 0x7f807f80u) + 0x00800080u) | ((w.y & 0x7f807f80u) + 0x00800080u)) |
          (((w.z & 0x7f807f80u) + 0x00800080u) | ((w.w & 0x7f807f80u) + 0x00800080u))) & 0x80008000u;
}

// Whether rows r0 .. r0 + 31 of the tile hold a value that is not finite, which its last plane tells (for
// the whole wave).
template <typename L, int ND>
__device__ __forceinline__ bool tile_not_finite(const u16* t, int r0) {
  stay_in_branch();
  uint32_t bad = 0;
#pragma unroll
  for (int s = 0; s < 2 * ND; ++s) {
    uint4 a[L::kPl];
    L::load_rows(t, r0, s, a);
    bad |= not_finite_bits(a[L::kPl - 1]);
  }
  return __ballot(bad != 0) != 0;
}

// A tensor's rows on their way to a tile of THREADS threads' workgroup: 16-byte vectors
// where rows allow them (width a multiple of a vector, base aligned), else entries.  Rows
// at and behind `rows` and columns at and behind the width read as zero.  A thread has
// one vector's place in a row, in every kPer-th row.
template <typename T, int ND, int ROWS, int THREADS, typename TILE = PairTile<T, ND, ROWS>>
struct TileStage {
  using L = TILE;
  static constexpr int kEV = 16 / sizeof(T);
  static constexpr int kU = L::kRow / kEV;  // vectors in a row
  static constexpr int kPer = THREADS / kU;
  static constexpr int kIt = (ROWS + kPer - 1) / kPer;
  static_assert(THREADS % kU == 0, "whole rows in a pass");
  const T* base;
  int rows, width, tid;
  bool vec;
  uint32_t off;
  VectorReader read;
  uint4 r[kIt];

  __device__ __forceinline__ void init(const T* p, int rows_, int width_, int tid_) {
    base = p, rows = rows_, width = width_, tid = tid_;
    vec = width % kEV == 0 && ((uintptr_t)p & 15) == 0;
    read = VectorReader(base, vec ? (int64_t)rows * width * (int)sizeof(T) : 0);
    const int row = tid / kU, col = tid % kU * kEV;
    off = col < width && row < ROWS ? (uint32_t)(row * width + col) * (uint32_t)sizeof(T) : kNoVector;
  }
  // the rows from r0 on
  template <bool STREAM = false>
  __device__ __forceinline__ void fetch(int r0) {
#pragma unroll
    for (int i = 0; i < kIt; ++i) {
      const uint32_t at = off + (uint32_t)(r0 + i * kPer) * (uint32_t)(width * (int)sizeof(T));
      r[i] = STREAM ? read.stream(at) : read(at);
    }
  }
  template <bool FAR>
  __device__ static __forceinline__ void put_planes(u16* dst, float f) {
#pragma unroll
    for (int i = 0; i < L::kPl; ++i) {
      const uint32_t b = pack2(FAR ? far_part(f, i) : f, 0.f);
      dst[i * L::kPlane] = (u16)b;
      f -= lo_f32(b);
    }
  }
  __device__ static void put_entry(u16* dst, T x) {
    if constexpr (sizeof(T) == 4) {
      put_planes<false>(dst, x);
      if (__builtin_expect(fabsf(x) > kLargestBf16, 0)) put_planes<true>(dst, x);  // (once more)
    } else {
      dst[0] = x;
    }
  }
  // FAR: some values of the vectors are beyond bfloat16's range
  template <bool FAR>
  __device__ __forceinline__ void put_vectors(u16* t) const {
#pragma unroll
    for (int i = 0; i < kIt; ++i) {
      const int row = tid / kU + i * kPer;
      if ((i + 1) * kPer > ROWS && row >= ROWS) continue;
      u16* const dst = t + L::at(row, tid % kU * kEV);
      if constexpr (sizeof(T) == 4) {
        float x[4] = {__uint_as_float(r[i].x), __uint_as_float(r[i].y), __uint_as_float(r[i].z), __uint_as_float(r[i].w)};
#pragma unroll
        for (int pl = 0; pl < L::kPl; ++pl) {
          auto part = [&](int j) { return FAR ? far_part(x[j], pl) : x[j]; };
          const uint2 b = {pack2(part(0), part(1)), pack2(part(2), part(3))};
          *(uint2*)(dst + pl * L::kPlane) = b;
          x[0] -= lo_f32(b.x), x[1] -= hi_f32(b.x), x[2] -= lo_f32(b.y), x[3] -= hi_f32(b.y);
        }
      } else {
        *(uint4*)dst = r[i];
      }
    }
  }
  __device__ __forceinline__ void put(u16* t, int r0) const {
    if (vec) {
      put_vectors<false>(t);
      if constexpr (sizeof(T) == 4) {
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < kIt; ++i) {
          most = fmaxf(fmaxf(most, fabsf(__uint_as_float(r[i].x))), fabsf(__uint_as_float(r[i].y)));
          most = fmaxf(fmaxf(most, fabsf(__uint_as_float(r[i].z))), fabsf(__uint_as_float(r[i].w)));
        }
        if (__builtin_expect(most > kLargestBf16, 0)) put_vectors<true>(t);  // (once more)
      }
    } else {
      if (put_entries<false>(t, r0) > kLargestBf16) put_entries<true>(t, r0);  // (once more)
    }
  }
  // the same entry by entry; the largest size (float32)
  template <bool FAR>
  __device__ __forceinline__ float put_entries(u16* t, int r0) const {
    float most = 0.f;
#pragma unroll 1
    for (int i = tid; i < ROWS * 32 * ND; i += THREADS) {
      const int row = i / (32 * ND), col = i % (32 * ND);
      const T x = r0 + row < rows && col < width ? base[(int64_t)(r0 + row) * width + col] : (T)0;
      if constexpr (sizeof(T) == 4) {
        put_planes<FAR>(t + L::at(row, col), x);
        most = fmaxf(most, fabsf(x));
      } else {
        put_entry(t + L::at(row, col), x);
      }
    }
    return most;
  }
};

// Two tensors x and y walked together, ROWS rows at a time, through LDS buffers of two tiles (x,
// then y) each: rows are fetched a whole step before they are put into the buffer that the step
// does not read.
template <typename T, int ND, int ROWS, int THREADS>
struct PairStage {
  using S = TileStage<T, ND, ROWS, THREADS>;
  using L = typename S::L;
  const T *x, *y;
  int x_width, y_width, rows, tid;
  S a, b;

  __device__ __forceinline__ void open(const T* x_, int x_width_, const T* y_, int y_width_, int rows_, int tid_) {
    x = x_, x_width = x_width_, y = y_, y_width = y_width_, rows = rows_, tid = tid_;
  }
  // both tensors' rows from r0 on, on their way
  __device__ __forceinline__ void fetch(int r0) {
    a.init(x, rows, x_width, tid);
    b.init(y, rows, y_width, tid);
    a.fetch(r0);
    b.fetch(r0);
  }
  // and there
  __device__ __forceinline__ void put(u16* buf, int r0) const {
    a.put(buf, r0);
    b.put(buf + L::kElems, r0);
  }
  __device__ __forceinline__ void load(u16* buf, int r0) {
    fetch(r0);
    put(buf, r0);
  }
  // work(buffer, r) for every 32 rows of a buffer, while the rows from `next` on (none where !more) go to `other`
  template <typename F>
  __device__ __forceinline__ void step(const u16* buf, u16* other, bool more, int next, F&& work) {
    if (more) fetch(next);
#pragma unroll 1
    for (int r = 0; r < ROWS; r += 32) work(buf, r);
    if (more) put(other, next);
  }
};

// A wave's own stores to LDS before its lanes' loads.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Right (or left) operands of one row per lane pair: entries 16 s + 8 h .. +7, all planes;
// zero past the width and where !ok.
template <int ND, bool FAR>
__device__ __forceinline__ float split_own32(const float* p, bool ok, int width, uint4 (&f)[2 * ND][3]) {
  const int h = (threadIdx.x & 63) >> 5;
  float most = 0.f;
#pragma unroll
  for (int s = 0; s < 2 * ND; ++s) {
    const int c0 = 16 * s + 8 * h;
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = ok && c0 + j < width ? p[c0 + j] : 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(x[j]));
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = FAR ? far_part(x[j], i) : x[j];
      f[s][i] = to_bf16(y);
      take_bf16(f[s][i], x);
    }
  }
  return most;
}
template <typename T, int ND>
__device__ __forceinline__ void load_own32(const T* p, bool ok, int width, uint4 (&f)[2 * ND][sizeof(T) == 4 ? 3 : 1]) {
  if constexpr (sizeof(T) == 4) {
    // (read once more where some are: a branch for every eight values would wait for each one's loads)
    if (__builtin_expect(split_own32<ND, false>(p, ok, width, f) > kLargestBf16, 0)) split_own32<ND, true>(p, ok, width, f);
  } else {
    const int h = (threadIdx.x & 63) >> 5;
    const bool vec = width % 8 == 0 && ((uintptr_t)p & 15) == 0;
#pragma unroll
    for (int s = 0; s < 2 * ND; ++s) {
      const int c0 = 16 * s + 8 * h;
      uint4 w = {0u, 0u, 0u, 0u};
      if (vec) {
        if (ok && c0 < width) w = *(const uint4*)(p + c0);
      } else {
        uint32_t u[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (ok && c0 + j < width) u[j >> 1] |= (uint32_t)p[c0 + j] << (16 * (j & 1));
        w = uint4{u[0], u[1], u[2], u[3]};
      }
      f[s][0] = w;
    }
  }
}

template <typename T>
__device__ __forceinline__ T rounded(float x) {
  if constexpr (sizeof(T) == 4) return x;
  else return (T)(pack2(x, 0.f) & 0xffffu);
}

// Four values of a row, columns c0 .. +3 (those below the width).
template <typename T>
__device__ __forceinline__ void store4(T* p, int c0, int width, const float (&x)[4], bool vec) {
  if (vec) {
    if (c0 < width) {
      if constexpr (sizeof(T) == 4) *(float4*)(p + c0) = float4{x[0], x[1], x[2], x[3]};
      else *(uint2*)(p + c0) = uint2{pack2(x[0], x[1]), pack2(x[2], x[3])};
    }
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (c0 + r < width) p[c0 + r] = rounded<T>(x[r]);
  }
}
// A lane's part of one output row: columns 32 j + 8 i + 4 h .. +3 of results acc[j], scaled,
// or zeros.
template <typename T, int ND>
__device__ __forceinline__ void store_row32(T* p, int width, const f32x16 (&acc)[ND], float scale, bool zero) {
  const int h = (threadIdx.x & 63) >> 5;
  const bool vec = width % 4 == 0 && ((uintptr_t)p & (4 * sizeof(T) - 1)) == 0;
#pragma unroll
  for (int j = 0; j < ND; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float x[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) x[r] = zero ? 0.f : acc[j][4 * i + r] * scale;
      store4(p, 32 * j + 8 * i + 4 * h, width, x, vec);
    }
}

// The sums of a workgroup's four waves with the same rows, in the waves' order: x[j] has columns 32 j + 8 wave + 4 h
// .. +3 of this lane's row.  buf: 1024 ND float4 of LDS that no wave reads any more when all
// have come here.
template <int ND>
__device__ __forceinline__ void join_waves(const f32x16 (&acc)[ND], float4* buf, float (&x)[ND][4]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < ND; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      buf[((wave * ND + j) * 4 + i) * 64 + lane] = float4{acc[j][4 * i], acc[j][4 * i + 1], acc[j][4 * i + 2], acc[j][4 * i + 3]};
  __syncthreads();
#pragma unroll
  for (int j = 0; j < ND; ++j) {
    x[j][0] = x[j][1] = x[j][2] = x[j][3] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float4 y = buf[((w * ND + j) * 4 + wave) * 64 + lane];
      x[j][0] += y.x, x[j][1] += y.y, x[j][2] += y.z, x[j][3] += y.w;
    }
  }
}
// A lane's part of an output row so joined, scaled, or zeros.
template <typename T, int ND>
__device__ __forceinline__ void store_joined(T* p, int width, float (&x)[ND][4], float scale, bool zero) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool vec = width % 4 == 0 && ((uintptr_t)p & (4 * sizeof(T) - 1)) == 0;
#pragma unroll
  for (int j = 0; j < ND; ++j) {
#pragma unroll
    for (int r = 0; r < 4; ++r) x[j][r] = zero ? 0.f : x[j][r] * scale;
    store4(p, 32 * j + 8 * wave + 4 * (lane >> 5), width, x[j], vec);
  }
}

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// v_exp_f32: within 1 ulp, results below 2^-126 are zero.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Whether `heads` heads of n tokens make so few workgroups of 128 rows that sweeps are the longest thing in the
// call, and a workgroup for every 32 rows, whose waves share one sweep, is faster.  Prompts / gradients in us,
// that way and with workgroups of 128 rows or more (on one card in turn), bfloat16 unless said: d = 64, 16 heads of
// 1000 tokens 13.6 / 35 and 20.2 / 58, 16 of 2000 29 / 76 and 34 / 102, 32 of 2000 50 / 140 and 36 / 118; d = 128, 1 of
// 8000 86 / 241 and 168 / 592, 16 of 1000 23 / 62 and 30 / 95, 16 of 2000 62 / 178 and 51 / 169, 128 of 128
// 12.8 / 37 and 11.0 / 30; float32, d = 64, 16 of 1000 41 / 118 and 60 / 162, 16 of 2000 119 / 345 and 108 / 300.
template <typename T, int ND>
inline bool few_sweeps(int64_t heads, int n) {
  return n > 128 && heads * ((n + 127) / 128) <= (sizeof(T) == 2 && ND <= 2 ? 256 : 128);
}

// Whether a bfloat16 call's workgroups take 256 rows, with eight waves, instead of 128: a staged tile serves
// twice as many rows, but there have to be two rounds of workgroups for the card.  Prompts in us with eight
// and four waves (on one card in turn), d = 128: 32 heads of 8192 tokens (1024 workgroups) 569 and 608, 64 of 2000
// (512) 89 and 91, 32 of 2000 (256) 66 and 57; gradients, rows of 256 and 128: 2255 and 2305, 336 and 339, 198 and 193.
inline bool eight_waves(int64_t heads, int n) { return heads * ((n + 255) / 256) >= 512; }

// Workgroups go to the 8 XCDs in turn.  With 8 heads or more each XCD takes whole
// heads, so that a head's rows are read through one L2, in sets of as many heads as make
// two rounds of workgroups on its 32 compute units: block by block within a set, so that a
// set ends with short sweeps everywhere (one head after the other left a third of the units
// idle at the end: n = 4096, 16 blocks, 4 heads an XCD, gradients 784 -> 662 us), and one
// after the other, so that few heads' rows compete for the L2.
__device__ __forceinline__ bool locate(int heads, int blocks, int& head, int& blk) {
  if (heads >= 8) {
    const int each = (heads + 7) >> 3, set = min(each, max(1, 64 / blocks));
    const int j = blockIdx.x >> 3, base = j / (set * blocks) * set, r = j - base * blocks, now = min(set, each - base);
    head = (base + r % now) * 8 + (int)(blockIdx.x & 7);
    blk = r / now;
    return head < heads;
  }
  head = blockIdx.x % heads;
  blk = blockIdx.x / heads;
  return true;
}
inline int64_t head_blocks(int heads, int blocks) {
  return (int64_t)blocks * (heads >= 8 ? ((int64_t)heads + 7) / 8 * 8 : heads);
}

__device__ __forceinline__ int tokens_of(const int* lengths, int b, int n) {
  return lengths ? min(max(lengths[b], 0), n) : n;
}

}  // namespace sata
