// Rotary positions: the pairs of the first 2 R entries of a head's row turned by the angle position times the
// pair's frequency,
//     (a, b) -> s (a cos x - b sin x, b cos x + a sin x),
// entries behind them as they are; back: by minus the angle (the transposed map, for gradients).
//
// Bound: memory, each row read and written once.  A thread has one vector's place in a row (of pairs
// whose partners lie R entries on: two vectors) and goes over up to 8 heads of its token with it, so that angle,
// sine and cosine (some 80 vector instructions a pair, a part of them in 64 bits) are formed once for
// them: no table of them in memory.  (Fewer heads where the card would not be full otherwise: at 12 heads of 3 x 2111 tokens, d =
// 80, each head forms its own, and its 24 MB take 9.8 us, twice a copy's time.)  In place too: nobody else reads what a thread writes.
// 40 heads of 4 x 4096 tokens, d = 128, bfloat16 (336 MB): 62.5 us, 5.4 TB/s.
//
// Precision: an angle is position times frequency in 64 bits, in turns, and only what is left of
// whole turns goes on in 32: positions of 2^21 lose nothing.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_common.hpp"
#include "kernels.hpp"
#include "series.hpp"

namespace sata {

namespace {

constexpr int kRotaryThreads = 256;
constexpr int kAhead = 4;  // heads whose rows are on their way at once

template <typename T, int V>
struct alignas(sizeof(T) * V) Entries {
  T x[V];
};
__device__ __forceinline__ float f32_of(float x) { return x; }
__device__ __forceinline__ float f32_of(u16 x) { return __uint_as_float((uint32_t)x << 16); }
template <typename T>
__device__ __forceinline__ T entry_from(float x) {
  if constexpr (sizeof(T) == 4) return x;
  else return (T)(pack2(x, 0.f) & 0xffffu);
}

// V: entries of a vector.  INTER: a place is V entries, V / 2 pairs of neighbours.  Otherwise place i is the V pairs
// i V .. +V-1 (i < R / V) or V entries that are copied; with V = 1, for rows that vectors of two do not fit, a
// pair's partner may be its neighbour.
template <typename T, int V, bool INTER>
__global__ void __launch_bounds__(kRotaryThreads) rotary_kernel(RotaryArgs a, int places, int each) {
  const int heads = a.Hq + a.Hk, h0 = blockIdx.y * each, h1 = min(heads, h0 + each);
  const int64_t all = (int64_t)a.B * a.n * places;
  for (int64_t at = (int64_t)blockIdx.x * kRotaryThreads + threadIdx.x; at < all; at += (int64_t)gridDim.x * kRotaryThreads) {
    const int64_t token = at / places;
    const int place = (int)(at - token * places), turned = INTER ? places : a.pairs / V;
    const int b = (int)(token / a.n), t = (int)(token - (int64_t)b * a.n);
    const bool turns = place < turned && (!INTER || place * (V / 2) < a.pairs);
    const bool next = V == 1 && a.interleaved;  // (the partner)
    const int partner = next ? 1 : a.pairs;
    const int col = INTER || place < turned ? place * (next ? 2 : V) : 2 * a.pairs + (place - turned) * V;
    constexpr int kPairs = INTER ? (V + 1) / 2 : V;
    float c[kPairs], s[kPairs];
    if (turns) {
      const double position = a.positions[token];
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const int p = place * kPairs + i;
        const bool in = p < a.pairs;
        const double x = position * ((double)a.freq[in ? p : 0] * 0.15915494309189533577);  // turns
        float si, co;
        sincospif(2.f * (float)(x - rint(x)), &si, &co);
        c[i] = co * a.scale;
        s[i] = (a.back ? -si : si) * a.scale;
      }
    }
    auto row_of = [&](const void* q, const void* k, int h) {
      const bool is_q = h < a.Hq;
      const int64_t row = ((int64_t)b * (is_q ? a.Hq : a.Hk) + (is_q ? h : h - a.Hq)) * a.n + t;
      return (const T*)(is_q ? q : k) + row * a.d;
    };
    using E = Entries<T, V>;
    for (int h = h0; h < h1; h += kAhead) {
      E x[kAhead], y[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (h + j < h1) {
          const T* const row = row_of(a.q, a.k, h + j);
          x[j] = *(const E*)(row + col);
          if constexpr (!INTER)
            if (turns) y[j] = *(const E*)(row + col + partner);
        }
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (h + j < h1) {
          T* const row = (T*)row_of(a.q_out, a.k_out, h + j);
          if (turns) {
            if constexpr (INTER) {
#pragma unroll
              for (int i = 0; i < kPairs; ++i) {
                const float u = f32_of(x[j].x[2 * i]), w = f32_of(x[j].x[2 * i + 1]);
                const T p = entry_from<T>(fmaf(u, c[i], -(w * s[i]))), r = entry_from<T>(fmaf(w, c[i], u * s[i]));
                const bool in = place * kPairs + i < a.pairs;
                x[j].x[2 * i] = in ? p : x[j].x[2 * i];
                x[j].x[2 * i + 1] = in ? r : x[j].x[2 * i + 1];
              }
            } else {
#pragma unroll
              for (int i = 0; i < kPairs; ++i) {
                const float u = f32_of(x[j].x[i]), w = f32_of(y[j].x[i]);
                x[j].x[i] = entry_from<T>(fmaf(u, c[i], -(w * s[i])));
                y[j].x[i] = entry_from<T>(fmaf(w, c[i], u * s[i]));
              }
              *(E*)(row + col + partner) = y[j];
            }
          }
          *(E*)(row + col) = x[j];
        }
    }
  }
}

template <typename T, int V, bool INTER>
hipError_t launch(const RotaryArgs& a, hipStream_t st) {
  const int places = INTER ? (a.d + V - 1) / V : a.pairs / V + (a.d - 2 * a.pairs) / V;
  const int heads = a.Hq + a.Hk;
  const int64_t units = (int64_t)a.B * a.n * places, blocks = (units + kRotaryThreads - 1) / kRotaryThreads;
  // As many heads a thread as leave the card 8 waves a SIMD, 8 at most.
  const int each = (int)std::min<int64_t>(8, std::max<int64_t>(1, blocks * heads / 2048));
  const int parts = (heads + each - 1) / each;  // (a launch has fewer than 2^32 threads)
  hipLaunchKernelGGL((rotary_kernel<T, V, INTER>), dim3((unsigned)std::min<int64_t>(blocks, (1 << 23) / parts), parts),
                     dim3(kRotaryThreads), 0, st, a, places, each);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_t(const RotaryArgs& a, hipStream_t st) {
  uintptr_t bits = (uintptr_t)a.q | (uintptr_t)a.q_out;
  if (a.Hk) bits |= (uintptr_t)a.k | (uintptr_t)a.k_out;
  // The widest vector (16 bytes at most) that rows, halves and tensors are whole multiples of.
  auto fits = [&](int v) {
    return a.d % v == 0 && (a.interleaved || a.pairs % v == 0) && bits % (v * sizeof(T)) == 0;
  };
  if (a.interleaved) {
    if (sizeof(T) == 2 && fits(8)) return launch<T, 8 / (sizeof(T) / 2), true>(a, st);
    if (fits(4)) return launch<T, 4, true>(a, st);
    if (fits(2)) return launch<T, 2, true>(a, st);
    return launch<T, 1, false>(a, st);
  }
  if (sizeof(T) == 2 && fits(8)) return launch<T, 8 / (sizeof(T) / 2), false>(a, st);
  if (fits(4)) return launch<T, 4, false>(a, st);
  if (fits(2)) return launch<T, 2, false>(a, st);
  return launch<T, 1, false>(a, st);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? launch_t<u16>(a, s) : launch_t<float>(a, s);
}

}  // namespace sata
