// Rows of a cache of 4 bits an entry.  Groups of 32 entries share a scale and a least value in bfloat16; an entry
// stands for least + scale * code.  A row of G groups (1, 2 or 4 with empty ones) is 20 G bytes:
// byte a G + g, a = 0..15, holds entry 32 g + a in its low and 32 g + 16 + a in its high four bits; then
// each group's scale and least value.  So the bytes of one a lie together: a lane of 16 has a column
// of every 16 in what it reads at once, and four lanes of keys' 16 bytes are a whole group's contraction.
//
// scale = (most - least) / 15, least the smallest entry, both rounded to bfloat16; codes are the nearest, to those
// rounded numbers, ties to the even one.  A group with an entry that is not finite, or beyond 2^120 in size (what
// softmax_step_packed.hip can still take sums of), stands for NaN.
#pragma once

#include <hip/hip_runtime.h>

#include "device_common.hpp"
#include "series.hpp"

namespace sata {

// scale (low half) and least value (high half) of a group with these extremes; `fine`: all entries are in range
__device__ __forceinline__ uint32_t group_params(float least, float most, bool fine) {
  // (halves: as written down for programs that form such rows on their own; no difference of them overflows.  The nearest
  // float32 to 1 / 7.5, not a division: torch multiplies too where a program on the GPU divides by a number)
  return fine ? pack2((0.5f * most - 0.5f * least) * (1.f / 7.5f), least) : 0x7fc07fc0u;
}
// What the codes of a group's entries take: (x / 2 - least / 2) / (scale / 2) as float32 division rounds it, then to the nearest.
// 1 / (scale / 2) is rounded to the nearest by one Newton step (of all 128 significands of a bfloat16, from any start two
// units off), so that a quotient and one correction give the nearest quotient too, but for scales so small that the
// correction's rest would not be a normal number: those divide.
struct GroupCode {
  float half, low, inverse;
  bool divide;
  __device__ __forceinline__ explicit GroupCode(uint32_t params) {
    half = 0.5f * lo_f32(params), low = 0.5f * hi_f32(params);
    const float r = __builtin_amdgcn_rcpf(half);
    inverse = fmaf(fmaf(-half, r, 1.f), r, r);
    divide = half < 0x1p-90f;
  }
  __device__ __forceinline__ uint32_t operator()(float x) const {
    const float a = 0.5f * x - low;
    float q = a * inverse;
    q = fmaf(fmaf(-q, half, a), inverse, q);
    if (__builtin_expect(divide, 0)) q = a / half;
    // (a scale of zero or NaN is not above zero)
    return half > 0.f ? (uint32_t)fminf(fmaxf(rintf(q), 0.f), 15.f) : 0u;
  }
};
__device__ __forceinline__ float value_of(uint32_t code, uint32_t params) {
  return fmaf((float)code, lo_f32(params), hi_f32(params));
}

// The least and the most of 16 lanes' values.
template <int CTRL>
__device__ __forceinline__ float turned_row(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ void ends_of_row(float& least, float& most) {
  least = fminf(least, turned_row<0x128>(least)), most = fmaxf(most, turned_row<0x128>(most));  // by 8, 4, 2, 1 lanes
  least = fminf(least, turned_row<0x124>(least)), most = fmaxf(most, turned_row<0x124>(most));
  least = fminf(least, turned_row<0x122>(least)), most = fmaxf(most, turned_row<0x122>(most));
  least = fminf(least, turned_row<0x121>(least)), most = fmaxf(most, turned_row<0x121>(most));
}
// What an entry counts as for a group's ends: one out of range as infinity, which tells.
__device__ __forceinline__ float for_ends(float x) { return fabsf(x) <= 0x1p120f ? x : INFINITY; }

// 16 lanes with the entries 32 g + a and 32 g + 16 + a of a row of width d, a = the lane: this lane's G bytes of codes,
// and the groups' scales and least values (the same in all lanes).
template <int G, typename F>
__device__ __forceinline__ uint32_t pack_row(int a, int d, F&& entry, uint32_t (&params)[G]) {
  uint32_t codes = 0;
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int i = 32 * g + a, j = i + 16;
    const float x = i < d ? entry(i) : 0.f, y = j < d ? entry(j) : 0.f;
    float least = i < d ? for_ends(x) : INFINITY, most = i < d ? for_ends(x) : -INFINITY;
    if (j < d) least = fminf(least, for_ends(y)), most = fmaxf(most, for_ends(y));
    ends_of_row(least, most);
    params[g] = 32 * g < d ? group_params(least, most, most < INFINITY) : 0u;
    const GroupCode code(params[g]);
    codes |= ((i < d ? code(x) : 0u) | (j < d ? code(y) : 0u) << 4) << (8 * g);
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
