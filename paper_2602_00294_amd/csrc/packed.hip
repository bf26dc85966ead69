// Rows into caches of 4 bits an entry, and back out of them as the values they stand for.
//
// Bound: memory, 2 or 4 bytes an entry on one side and 5 bits on the other.  A lane has a group of 32 entries, which it reads or
// writes by whole vectors, and finds their ends and codes without another; the row's bytes, of which each group has every
// G-th, change lanes (DPP) and places (v_perm) once.
// Keys and values of 32 heads x 4000 rows of 128 bfloat16 entries (86 MB): written in 16.8 us, of which vector
// instructions take 92% (a lane's division and rounding of 32 entries; 16 lanes to a group, as a token's row
// is packed, took 36); read back in 15.8 us each.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "kernels.hpp"
#include "packed_rows.hpp"

namespace sata {

namespace {

constexpr int kPackThreads = 256;

__device__ __forceinline__ float f32_of(float x) { return x; }
__device__ __forceinline__ float f32_of(u16 x) { return __uint_as_float((uint32_t)x << 16); }

template <int CTRL>
__device__ __forceinline__ uint32_t neighbour(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
// One of four dwords.
__device__ __forceinline__ uint32_t pick(const uint32_t (&x)[4], int i) {
  const uint32_t a = i & 1 ? x[1] : x[0], b = i & 1 ? x[3] : x[2];
  return i & 2 ? b : a;
}
// Four lanes with four dwords each: lane l's i-th becomes lane i's l-th.
__device__ __forceinline__ void across_four(uint32_t (&x)[4], int l) {
  uint32_t y[4];
  y[0] = pick(x, l);
  y[1] = neighbour<0xb1>(pick(x, l ^ 1));  // lanes 1, 0, 3, 2
  y[2] = neighbour<0x4e>(pick(x, l ^ 2));  // 2, 3, 0, 1
  y[3] = neighbour<0x1b>(pick(x, l ^ 3));  // 3, 2, 1, 0
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = pick(y, l ^ i);
}
// Byte j of dword i becomes byte i of dword j.
__device__ __forceinline__ void across_bytes(uint32_t (&x)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(x[1], x[0], 0x05010400), b = __builtin_amdgcn_perm(x[1], x[0], 0x07030602);
  const uint32_t c = __builtin_amdgcn_perm(x[3], x[2], 0x05010400), d = __builtin_amdgcn_perm(x[3], x[2], 0x07030602);
  x[0] = __builtin_amdgcn_perm(c, a, 0x05040100), x[1] = __builtin_amdgcn_perm(c, a, 0x07060302);
  x[2] = __builtin_amdgcn_perm(d, b, 0x05040100), x[3] = __builtin_amdgcn_perm(d, b, 0x07060302);
}
// A group's 16 bytes, dword w of a = 4 w .. +3, from the 16 bytes that this lane has of its row (lane g of G: of a = 16 g / G on), or
// the other way (TO_ROW).
template <int G, bool TO_ROW>
__device__ __forceinline__ void change_places(uint32_t (&x)[4], int g) {
  if constexpr (G == 4) {
    if (TO_ROW) across_four(x, g);
    across_bytes(x);
    if (!TO_ROW) across_four(x, g);
  } else if constexpr (G == 2) {
    if constexpr (TO_ROW) {
      // (the other lane's dwords of this lane's a)
      const uint32_t a = neighbour<0xb1>(g ? x[0] : x[2]), b = neighbour<0xb1>(g ? x[1] : x[3]);
      const uint32_t own0 = g ? x[2] : x[0], own1 = g ? x[3] : x[1];
      const uint32_t f0 = g ? a : own0, s0 = g ? own0 : a, f1 = g ? b : own1, s1 = g ? own1 : b;  // of groups 0 and 1
      x[0] = __builtin_amdgcn_perm(s0, f0, 0x05010400), x[1] = __builtin_amdgcn_perm(s0, f0, 0x07030602);
      x[2] = __builtin_amdgcn_perm(s1, f1, 0x05010400), x[3] = __builtin_amdgcn_perm(s1, f1, 0x07030602);
    } else {
      const uint32_t f0 = __builtin_amdgcn_perm(x[1], x[0], 0x06040200), s0 = __builtin_amdgcn_perm(x[1], x[0], 0x07050301);
      const uint32_t f1 = __builtin_amdgcn_perm(x[3], x[2], 0x06040200), s1 = __builtin_amdgcn_perm(x[3], x[2], 0x07050301);
      const uint32_t a = neighbour<0xb1>(g ? f0 : s0), b = neighbour<0xb1>(g ? f1 : s1);
      if (g) x[0] = a, x[1] = b, x[2] = s0, x[3] = s1;
      else x[0] = f0, x[1] = f1, x[2] = a, x[3] = b;
    }
  }
}

template <typename T, int G, bool WRITE>
__device__ __forceinline__ void rows_of(const PackedArgs& p, const PackedRows& r) {
  constexpr int kEV = 16 / (int)sizeof(T), kRows = kPackThreads / G;
  const int g = threadIdx.x % G, d = r.d, left = d - 32 * g;  // entries from this group on
  const int64_t rows = (int64_t)p.heads * p.n;
  const bool vec = d % kEV == 0 && ((uintptr_t)r.x & 15) == 0;
  for (int64_t i = (int64_t)blockIdx.x * kRows + threadIdx.x / G; i < rows; i += (int64_t)gridDim.x * kRows) {
    const int64_t head = i / p.n;
    const int t = (int)(i - head * p.n), b = (int)(head / p.H);
    const int64_t at = (p.first ? (int64_t)p.first[b] : 0) + t;
    const bool there = at >= 0 && at < p.capacity && (!p.counts || t < p.counts[b]);
    uint8_t* const row = r.cache + (head * p.capacity + at) * (20 * G);
    T* const x = (T*)r.x + i * d + 32 * g;
    float f[32];
    uint32_t w[4], params = 0u;
    // 16 bytes of the row as it lies: rows of 80 bytes are aligned to 16, of 40 to 8, of 20 to 4
    auto row_dwords = [&](auto&& each) {
      uint8_t* const q = row + 16 * g;
      if constexpr (G == 4) each((uint4*)q);
      else if constexpr (G == 2) each((uint2*)q);
      else each((uint32_t*)q);
    };
    if constexpr (WRITE) {
      if (!there) continue;  // (the same for the lanes of a row)
      if (vec) {
#pragma unroll
        for (int c = 0; c < 32; c += kEV) {
          uint4 v = {0u, 0u, 0u, 0u};
          if (c < left) v = *(const uint4*)(x + c);
          const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 2) f[c + 2 * e] = lo_f32(u[e]), f[c + 2 * e + 1] = hi_f32(u[e]);
            else f[c + e] = __uint_as_float(u[e]);
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < 32; ++e) f[e] = e < left ? f32_of(x[e]) : 0.f;
      }
      float least = INFINITY, most = -INFINITY;
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        const float y = for_ends(f[e]);
        least = fminf(least, e < left ? y : INFINITY), most = fmaxf(most, e < left ? y : -INFINITY);
      }
      params = left > 0 ? group_params(least, most, most < INFINITY) : 0u;
      const GroupCode code(params);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        w[q] = 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int lo = 4 * q + e, hi = lo + 16;
          w[q] |= ((lo < left ? code(f[lo]) : 0u) | (hi < left ? code(f[hi]) : 0u) << 4) << (8 * e);
        }
      }
      change_places<G, true>(w, g);
      row_dwords([&](auto* q) {
        using V = std::remove_pointer_t<decltype(q)>;
#pragma unroll
        for (int e = 0; e < 16 / (int)sizeof(V); ++e) {
          if constexpr (sizeof(V) == 16) q[e] = uint4{w[0], w[1], w[2], w[3]};
          else if constexpr (sizeof(V) == 8) q[e] = uint2{w[2 * e], w[2 * e + 1]};
          else q[e] = w[e];
        }
      });
      ((uint32_t*)(row + 16 * G))[g] = params;
    } else {
      w[0] = w[1] = w[2] = w[3] = 0u;
      if (there) {
        row_dwords([&](auto* q) {
          using V = std::remove_pointer_t<decltype(q)>;
#pragma unroll
          for (int e = 0; e < 16 / (int)sizeof(V); ++e) {
            const V v = q[e];
            if constexpr (sizeof(V) == 16) w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
            else if constexpr (sizeof(V) == 8) w[2 * e] = v.x, w[2 * e + 1] = v.y;
            else w[e] = v;
          }
        });
        params = ((const uint32_t*)(row + 16 * G))[g];
      }
      change_places<G, false>(w, g);
#pragma unroll
      for (int e = 0; e < 32; ++e) f[e] = value_of((w[(e & 15) / 4] >> (8 * (e & 3) + 4 * (e >> 4))) & 15u, params);
      if (vec) {
#pragma unroll
        for (int c = 0; c < 32; c += kEV) {
          uint4 v;
          if constexpr (sizeof(T) == 2) v = uint4{pack2(f[c], f[c + 1]), pack2(f[c + 2], f[c + 3]), pack2(f[c + 4], f[c + 5]), pack2(f[c + 6], f[c + 7])};
          else v = uint4{__float_as_uint(f[c]), __float_as_uint(f[c + 1]), __float_as_uint(f[c + 2]), __float_as_uint(f[c + 3])};
          if (c < left) *(uint4*)(x + c) = v;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 32; ++e)
          if (e < left) {
            if constexpr (sizeof(T) == 4) x[e] = f[e];
            else x[e] = (T)(pack2(f[e], 0.f) & 0xffffu);
          }
      }
    }
  }
}

template <typename T, bool WRITE>
__global__ void __launch_bounds__(kPackThreads) packed_kernel(PackedArgs p) {
  const PackedRows& r = p.rows[blockIdx.y];
  switch (packed_groups(r.d)) {
    case 1: return rows_of<T, 1, WRITE>(p, r);
    case 2: return rows_of<T, 2, WRITE>(p, r);
    default: return rows_of<T, 4, WRITE>(p, r);
  }
}

template <typename T, bool WRITE>
hipError_t launch(const PackedArgs& p, hipStream_t s) {
  const int d = p.tensors > 1 ? std::max(p.rows[0].d, p.rows[1].d) : p.rows[0].d, each = kPackThreads / packed_groups(d);
  const int64_t blocks = ((int64_t)p.heads * p.n + each - 1) / each;
  hipLaunchKernelGGL((packed_kernel<T, WRITE>), dim3((unsigned)std::min<int64_t>(blocks, 1 << 20), p.tensors),
                     dim3(kPackThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_write(const PackedArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? launch<u16, true>(a, s) : launch<float, true>(a, s);
}
hipError_t launch_packed_read(const PackedArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? launch<u16, false>(a, s) : launch<float, false>(a, s);
}

}  // namespace sata
