// Rows of a cache of 4 bits an entry.  Groups of 32 entries share a scale and a least value in bfloat16; an entry
// stands for least + scale * code.  A row of G groups (1, 2 or 4 with empty ones) is 20 G bytes:
// byte a G + g, a = 0..15, holds entry 32 g + a in its low and 32 g + 16 + a in its high four bits; then
// each group's scale and least value.  So the bytes of one a lie together: a lane of 16 has a column
// of every 16 in what it reads at once, and four lanes of keys' 16 bytes are a whole group's contraction.
//
// scale = (most - least) / 15, least the smallest entry, both rounded to bfloat16; codes are the nearest, to those
// rounded numbers, ties to the even one.  A group with an entry that is not finite, or beyond 2^120 in size (31
// scales have to be a number), stands for NaN.
#pragma once

#include <hip/hip_runtime.h>

#include "device_common.hpp"
#include "series.hpp"

namespace sata {

// scale (low half) and least value (high half) of a group with these extremes; `fine`: all entries are in range
__device__ __forceinline__ uint32_t group_params(float least, float most, bool fine) {
  // (halves: as written down for programs that form such rows on their own; no difference of them overflows)
  return fine ? pack2((0.5f * most - 0.5f * least) / 7.5f, least) : 0x7fc07fc0u;
}
__device__ __forceinline__ uint32_t code_of(float x, uint32_t params) {
  const float half = 0.5f * lo_f32(params), low = 0.5f * hi_f32(params);
  // (a scale of NaN is not above zero)
  return half > 0.f ? (uint32_t)fminf(fmaxf(rintf((0.5f * x - low) / half), 0.f), 15.f) : 0u;
}
__device__ __forceinline__ float value_of(uint32_t code, uint32_t params) {
  return fmaf((float)code, lo_f32(params), hi_f32(params));
}

// 16 lanes with the entries 32 g + a and 32 g + 16 + a of a row of width d, a = the lane: this lane's G bytes of codes,
// and the groups' scales and least values (the same in all lanes).
template <int G, typename F>
__device__ __forceinline__ uint32_t pack_row(int a, int d, F&& entry, uint32_t (&params)[G]) {
  uint32_t codes = 0;
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int i = 32 * g + a, j = i + 16;
    const float x = i < d ? entry(i) : 0.f, y = j < d ? entry(j) : 0.f;
    float least = i < d ? x : INFINITY, most = i < d ? x : -INFINITY;
    if (j < d) least = fminf(least, y), most = fmaxf(most, y);
    int fine = fabsf(x) <= 0x1p120f && fabsf(y) <= 0x1p120f;
#pragma unroll
    for (int m = 1; m < 16; m *= 2) {
      least = fminf(least, __shfl_xor(least, m));
      most = fmaxf(most, __shfl_xor(most, m));
      fine &= __shfl_xor(fine, m);
    }
    params[g] = 32 * g < d ? group_params(least, most, fine) : 0u;
    codes |= ((i < d ? code_of(x, params[g]) : 0u) | (j < d ? code_of(y, params[g]) : 0u) << 4) << (8 * g);
  }
  return codes;
}

// This lane's bytes of the row at p, and (lane a < G) a group's scale and least value.
template <int G>
__device__ __forceinline__ void store_packed(uint8_t* p, int a, uint32_t codes, const uint32_t (&params)[G]) {
  if constexpr (G == 4) ((uint32_t*)p)[a] = codes;
  else if constexpr (G == 2) ((uint16_t*)p)[a] = (uint16_t)codes;
  else p[a] = (uint8_t)codes;
#pragma unroll
  for (int g = 0; g < G; ++g)
    if (a == g) ((uint32_t*)(p + 16 * G))[g] = params[g];
}
template <int G>
__device__ __forceinline__ uint32_t load_packed(const uint8_t* p, int a) {
  if constexpr (G == 4) return ((const uint32_t*)p)[a];
  else if constexpr (G == 2) return ((const uint16_t*)p)[a];
  else return p[a];
}

}  // namespace sata
