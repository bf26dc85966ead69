// Rows into caches of 4 bits an entry, and back out of them as the values they stand for.
//
// Bound: memory, 2 or 4 bytes an entry on one side and 5 bits on the other.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kernels.hpp"
#include "packed_rows.hpp"

namespace sata {

namespace {

constexpr int kPackThreads = 256;

__device__ __forceinline__ float f32_of(float x) { return x; }
__device__ __forceinline__ float f32_of(u16 x) { return __uint_as_float((uint32_t)x << 16); }

// 16 lanes a row.
template <typename T, int G, bool WRITE>
__device__ __forceinline__ void rows_of(const PackedArgs& p, const PackedRows& r) {
  const int a = threadIdx.x & 15;
  const int64_t rows = (int64_t)p.heads * p.n;
  for (int64_t i = (int64_t)blockIdx.x * (kPackThreads / 16) + threadIdx.x / 16; i < rows;
       i += (int64_t)gridDim.x * (kPackThreads / 16)) {
    const int64_t head = i / p.n;
    const int t = (int)(i - head * p.n), b = (int)(head / p.H);
    const int64_t at = (p.first ? (int64_t)p.first[b] : 0) + t;
    const bool there = at >= 0 && at < p.capacity && (!p.counts || t < p.counts[b]);
    uint8_t* const row = r.cache + (head * p.capacity + at) * (20 * G);
    T* const x = (T*)r.x + i * r.d;
    if constexpr (WRITE) {
      if (!there) continue;  // (the same for the 16 lanes of a row)
      uint32_t params[G];
      const uint32_t codes = pack_row<G>(a, r.d, [&](int e) { return f32_of(x[e]); }, params);
      store_packed<G>(row, a, codes, params);
    } else {
      const uint32_t codes = there ? load_packed<G>(row, a) : 0u;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const uint32_t params = there ? ((const uint32_t*)(row + 16 * G))[g] : 0u;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int e = 32 * g + 16 * h + a;
          const float y = value_of((codes >> (8 * g + 4 * h)) & 15u, params);
          if (e < r.d) {
            if constexpr (sizeof(T) == 4) x[e] = y;
            else x[e] = (T)(pack2(y, 0.f) & 0xffffu);
          }
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
  const int64_t blocks = ((int64_t)p.heads * p.n + kPackThreads / 16 - 1) / (kPackThreads / 16);
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
