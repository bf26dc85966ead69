// Rows into caches of 4 bits an entry, and back out of them as the values they stand for.
//
// Bound: memory, 2 or 4 bytes an entry on one side and 5 bits on the other.  Writing, a lane has a group of 32 entries, which it
// reads by whole vectors, and finds their ends and codes without another; the row's bytes, of which each group has every
// G-th, change lanes (DPP) and places (v_perm) once.  Reading, a lane has eight entries and writes whole vectors side by
// side with its neighbours'.
// Keys and values of 32 heads x 4000 rows of 128 entries: bfloat16 (86 MB) written in 22.7 us, 3.8 TB/s, float32 (151 MB) in
// 32, 4.7 TB/s; half of the bfloat16 rows, as padded prompts have them (43 MB), in 17 to 18, of which vector
// instructions take 92% (a lane's division and rounding of 32 entries; 16 lanes to a group, as a token's row
// is packed, took 36); all read back in 10.3 us each, 4.2 TB/s (a lane a group, as they are written, took 15.8).
#include <hip/hip_runtime.h>

#include <algorithm>

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
// A group's 16 bytes, dword w of a = 4 w .. +3, become the 16 bytes that this lane, g of G, has of its row: of a = 16 g / G on.
template <int G>
__device__ __forceinline__ void to_row(uint32_t (&x)[4], int g) {
  if constexpr (G == 4) {
    across_four(x, g);
    across_bytes(x);
  } else if constexpr (G == 2) {
    // (the other lane's dwords of this lane's a)
    const uint32_t a = neighbour<0xb1>(g ? x[0] : x[2]), b = neighbour<0xb1>(g ? x[1] : x[3]);
    const uint32_t own0 = g ? x[2] : x[0], own1 = g ? x[3] : x[1];
    const uint32_t f0 = g ? a : own0, s0 = g ? own0 : a, f1 = g ? b : own1, s1 = g ? own1 : b;  // of groups 0 and 1
    x[0] = __builtin_amdgcn_perm(s0, f0, 0x05010400), x[1] = __builtin_amdgcn_perm(s0, f0, 0x07030602);
    x[2] = __builtin_amdgcn_perm(s1, f1, 0x05010400), x[3] = __builtin_amdgcn_perm(s1, f1, 0x07030602);
  }
}

template <typename T, int G>
__device__ __forceinline__ void write_rows(const PackedArgs& p, const PackedRows& r) {
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
    for (int i = 0; i < 4; ++i) {
      w[i] = 0u;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int lo = 4 * i + e, hi = lo + 16;
        w[i] |= ((lo < left ? code(f[lo]) : 0u) | (hi < left ? code(f[hi]) : 0u) << 4) << (8 * e);
      }
    }
    to_row<G>(w, g);
    uint8_t* const q = row + 16 * g;  // (rows of 80 bytes are aligned to 16, of 40 to 8, of 20 to 4)
    if constexpr (G == 4) {
      *(uint4*)q = uint4{w[0], w[1], w[2], w[3]};
    } else if constexpr (G == 2) {
      ((uint2*)q)[0] = uint2{w[0], w[1]}, ((uint2*)q)[1] = uint2{w[2], w[3]};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) ((uint32_t*)q)[e] = w[e];
    }
    ((uint32_t*)(row + 16 * G))[g] = params;
  }
}

template <typename T>
__global__ void __launch_bounds__(kPackThreads) packed_write_kernel(PackedArgs p) {
  const PackedRows& r = p.rows[blockIdx.y];
  switch (packed_groups(r.d)) {
    case 1: return write_rows<T, 1>(p, r);
    case 2: return write_rows<T, 2>(p, r);
    default: return write_rows<T, 4>(p, r);
  }
}

// Eight entries a lane: their bytes lie G apart in 8 G bytes, which the lanes of the other groups and halves read too.
template <typename T, int G>
__global__ void __launch_bounds__(kPackThreads) packed_read_kernel(PackedArgs p) {
  const PackedRows& r = p.rows[0];
  const int d = r.d, head = blockIdx.y;
  const uint32_t parts = (uint32_t)(d + 7) / 8, all = (uint32_t)p.n * parts;
  const bool vec = d % 8 == 0 && ((uintptr_t)r.x & 15) == 0;
  const int64_t first = p.first ? p.first[head / p.H] : 0;
  const uint8_t* const cache = r.cache + (int64_t)head * p.capacity * (20 * G);
  for (uint32_t i = blockIdx.x * kPackThreads + threadIdx.x; i < all; i += gridDim.x * kPackThreads) {
    const uint32_t t = i / parts;
    const int e0 = 8 * (int)(i - t * parts), g = e0 / 32, high = e0 % 32 / 16;
    const int64_t at = first + t;
    uint32_t w[2 * G] = {}, params = 0u;
    if (at >= 0 && at < p.capacity) {
      const uint8_t* const row = cache + at * (20 * G);
      const uint8_t* const q = row + e0 % 16 * G;  // (aligned as the row: to 16, 8 or 4 bytes)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        if constexpr (G == 4) {
          const uint4 v = ((const uint4*)q)[x];
          w[4 * x] = v.x, w[4 * x + 1] = v.y, w[4 * x + 2] = v.z, w[4 * x + 3] = v.w;
        } else if constexpr (G == 2) {
          const uint2 v = ((const uint2*)q)[x];
          w[2 * x] = v.x, w[2 * x + 1] = v.y;
        } else {
          w[x] = ((const uint32_t*)q)[x];
        }
      }
      params = ((const uint32_t*)(row + 16 * G))[g];
    }
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = value_of((w[e * G / 4] >> (8 * (e * G % 4 + g) + 4 * high)) & 15u, params);
    T* const x = (T*)r.x + ((int64_t)head * p.n + t) * d + e0;
    if (vec) {
      if constexpr (sizeof(T) == 2) {
        *(uint4*)x = uint4{pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7])};
      } else {
        ((float4*)x)[0] = float4{f[0], f[1], f[2], f[3]};
        ((float4*)x)[1] = float4{f[4], f[5], f[6], f[7]};
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e0 + e < d) {
          if constexpr (sizeof(T) == 4) x[e] = f[e];
          else x[e] = (T)(pack2(f[e], 0.f) & 0xffffu);
        }
    }
  }
}

template <typename T>
hipError_t launch_write(const PackedArgs& p, hipStream_t s) {
  const int d = p.tensors > 1 ? std::max(p.rows[0].d, p.rows[1].d) : p.rows[0].d, each = kPackThreads / packed_groups(d);
  const int64_t blocks = ((int64_t)p.heads * p.n + each - 1) / each;
  hipLaunchKernelGGL((packed_write_kernel<T>), dim3((unsigned)std::min<int64_t>(blocks, 1 << 20), p.tensors), dim3(kPackThreads), 0, s, p);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_read(const PackedArgs& p, hipStream_t s) {
  const int64_t blocks = ((int64_t)p.n * ((p.rows[0].d + 7) / 8) + kPackThreads - 1) / kPackThreads;
  // (a launch has fewer than 2^32 threads)
  const dim3 grid((unsigned)std::min<int64_t>(blocks, (1 << 23) / p.heads), p.heads);
  switch (packed_groups(p.rows[0].d)) {
    case 1: hipLaunchKernelGGL((packed_read_kernel<T, 1>), grid, dim3(kPackThreads), 0, s, p); break;
    case 2: hipLaunchKernelGGL((packed_read_kernel<T, 2>), grid, dim3(kPackThreads), 0, s, p); break;
    default: hipLaunchKernelGGL((packed_read_kernel<T, 4>), grid, dim3(kPackThreads), 0, s, p); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_write(const PackedArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? launch_write<u16>(a, s) : launch_write<float>(a, s);
}
hipError_t launch_packed_read(const PackedArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? launch_read<u16>(a, s) : launch_read<float>(a, s);
}

}  // namespace sata
