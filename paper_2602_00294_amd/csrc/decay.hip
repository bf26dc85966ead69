// Causal linear attention with a decay per head: with lam = exp(log_decay[h]) and
// c = 1 / sqrt(d_k),
//     S_t = lam S_{t-1} + k_t (x) v_t,   y_t = c q_t S_t,
// and its gradients.  All four sums over a sequence (y, dq, dk and
// dv) are one scan with the tensors in other places,
//     out_t = c sum_{s<=t} lam^(t-s) (a_t . b_s) w_s + (the state before the first token),
//     y : a = q,  b = k,  w = v         dq: a = dy, b = v,  w = k
//     dv: a = k,  b = q,  w = dy        dk: a = v,  b = dy, w = q   (from the last token back)
#include <hip/hip_runtime.h>

#include <algorithm>

#include "decay_power.hpp"
#include "device_common.hpp"
#include "kernels.hpp"
#include "pair_tiles.hpp"

namespace sata {

namespace {

// A stretch of one head's tokens per workgroup, in chunks of kChunk, the state in
// registers: wave j holds columns 32 j .. +31 of it (and writes those of the output), its lanes one
// column each.  With r a row of a chunk of m tokens and R the state before it (forward)
//     out_r = readout lam^(r+1) a_r R + sum_{s<=r} update readout lam^(r-s) (a_r.b_s) w_s
//     R     = lam^m R + sum_s update lam^(m-1-s) b_s (x) w_s
// and in reverse the same with lam^(m-1-r), lam^(s-r) and lam^(s+1).
//
// Precision: bfloat16 inputs are exact operands; the pairs' weights are rounded to
// bfloat16 as the output is; the state is read out as two bfloat16 numbers and what is
// added to it carries 24 bits (w times its power as three), so that the state is a float32 one.
// float32 inputs, weights and states: three bfloat16 numbers each.
constexpr int kChunk = 32;

struct ScanParts {
  int parts, part_len;  // stretches per head, tokens in each (a multiple of the chunk)
  float* states;        // [heads][parts][da][dw]: what each adds (written) or starts from (read); null: one part
};

// Entries 16 s + 4 h .. +3 and 16 s + 8 + 4 h .. +3 of rows r0 .. r0 + 31: the order of a result's
// numbers, so that the state contracts with these rows as it lies in its registers.
template <typename L>
__device__ __forceinline__ void load_rows_as_results(const u16* t, int r0, int s, uint4 (&op)[L::kPl]) {
  const int lane = threadIdx.x & 63, l31 = lane & 31, h = lane >> 5;
  const u16* const row = t + (r0 + l31) * L::kRow + 4 * h;
  const u16* const a = row + 8 * ((2 * s) ^ L::swap(l31));
  const u16* const b = row + 8 * ((2 * s + 1) ^ L::swap(l31));
#pragma unroll
  for (int i = 0; i < L::kPl; ++i) {
    const uint2 x = *(const uint2*)(a + i * L::kPlane), y = *(const uint2*)(b + i * L::kPlane);
    op[i] = uint4{x.x, x.y, y.x, y.y};
  }
}

// REV: from the last token back.  The members of a group (G) vary in a forward, and in b
// and w in reverse.  SUMS: only what the part adds to the state, from zero.
template <typename T, int ND, bool REV, bool SUMS>
__global__ void __launch_bounds__(64 * ND, sizeof(T) == 2 ? 2 : 1) decay_scan_kernel(DecayScan s, ScanParts p) {
  constexpr int C = kChunk, kThreads = 64 * ND, kTiles = C / 32;
  using L = PairTile<T, ND, C>;
  constexpr int PS = sizeof(T) == 2 ? 2 : 3;  // numbers of a state's entry in its readout
  extern __shared__ __attribute__((aligned(16))) u16 smem16[];
  u16* const ta = smem16;
  u16* const tb = smem16 + L::kElems;
  u16* const tw = smem16 + 2 * L::kElems;
  // lam^0 .. lam^C, behind C zeros (a power's place is a lane's number plus a constant)
  float* const power = (float*)(smem16 + 3 * L::kElems) + C;
  const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
  const int len = tokens_of(s.lengths, head / s.H, s.n);
  const int first = part * p.part_len, last = min(first + p.part_len, s.n), end = max(first, min(last, len));
  const int chunks = (end - first + C - 1) / C;
  const int col = 32 * wave + l31;
  const float rate = s.log_decay[head % s.H];
  for (int e = tid; e <= C; e += kThreads) {
    power[e] = decay_power(rate, e).hi;
    if (e > 0) power[-e] = 0.f;
  }
  // (only the chunk at the sequence's end has fewer tokens)
  const FloatPair whole = decay_power(rate, C), tail = decay_power(rate, end - first - (chunks - 1) * C);

  f32x16 S[ND];
  auto state_at = [&](int j, int i, bool transposed) {
    const int r = 32 * j + result_row(i, h);
    return transposed ? (int64_t)col * s.da + r : (int64_t)r * s.dw + col;
  };
  auto has = [&](int j, int i) { return 32 * j + result_row(i, h) < s.da && col < s.dw; };
  const int64_t size = (int64_t)s.da * s.dw;
  const float* const from = SUMS ? nullptr : p.states ? p.states + ((int64_t)head * p.parts + part) * size
                                           : s.S_in ? s.S_in + head * size : nullptr;
#pragma unroll
  for (int j = 0; j < ND; ++j)
#pragma unroll
    for (int i = 0; i < 16; ++i) S[j][i] = from && has(j, i) ? from[state_at(j, i, !p.states && s.transposed)] : 0.f;

  if (chunks > 0) {
    const int G = SUMS && !REV ? 1 : s.G, units = chunks * G;
    TileStage<T, ND, C, kThreads> sa, sb, sw;
    auto row_of = [&](int c) { return first + (REV ? chunks - 1 - c : c) * C; };
    // tiles that unit (c, g) needs anew
    auto new_a = [&](int g) { return !SUMS && (!REV || g == 0); };
    auto new_b = [&](int g) { return REV || g == 0; };
    auto fetch = [&](int g, int t0) {
      if (new_a(g)) {
        sa.init((const T*)s.a + ((int64_t)head * (REV ? 1 : s.G) + (REV ? 0 : g)) * s.n * s.da, len, s.da, tid);
        sa.fetch(t0);
      }
      if (new_b(g)) {
        const int64_t m = (int64_t)head * (REV ? s.G : 1) + (REV ? g : 0);
        sb.init((const T*)s.b + m * s.n * s.da, len, s.da, tid);
        sw.init((const T*)s.w + m * s.n * s.dw, len, s.dw, tid);
        sb.fetch(t0);
        sw.fetch(t0);
      }
    };
    const float scale = s.update * s.readout;
    fetch(0, row_of(0));
    f32x16 o[kTiles];
    for (int u = 0, c = 0, g = 0; u < units; ++u) {
      const int t0 = row_of(c), m = min(C, end - t0);
      const bool opens = g == 0, closes = g + 1 == G;
      __syncthreads();  // the tiles were last read before this
      if (new_a(g)) sa.put(ta, t0);
      if (new_b(g)) {
        sb.put(tb, t0);
        sw.put(tw, t0);
      }
      __syncthreads();
      const int member = g;
      if (closes) g = 0, ++c;
      else ++g;
      if (u + 1 < units) fetch(g, row_of(c));

      auto early = [&](int r) { return power[r + 1]; };
      auto late = [&](int r) { return power[m - 1 - r]; };
      // this wave's columns of w: operands of rows 16 x .. +15
      uint4 wf[C / 16][L::kPl];
      uint32_t bad = 0;
#pragma unroll
      for (int x = 0; x < C / 16; ++x) {
        L::load_transposed(tw, 16 * x, wave, wf[x]);
        const uint4 b = not_finite_entries(wf[x][0]);
        bad |= b.x | b.y | b.z | b.w;
      }
      if constexpr (!SUMS) {
        if (!REV || opens) {
#pragma unroll
          for (int q = 0; q < kTiles; ++q) o[q] = zero16();
#pragma unroll
          for (int x = 0; x < 2 * ND; ++x) {
            float v[8];
            uint4 st[1][PS];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = S[x / 2][8 * (x & 1) + i];
            to_planes<PS>(v, st);
#pragma unroll
            for (int q = 0; q < kTiles; ++q) {
              uint4 f[L::kPl];
              load_rows_as_results<L>(ta, 32 * q, x, f);
              o[q] = dot_planes32(st[0], f, o[q]);
            }
          }
#pragma unroll
          for (int q = 0; q < kTiles; ++q) {
            const int r = 32 * q + l31;
            const float k = s.readout * (REV ? late(r) : early(r));
#pragma unroll
            for (int i = 0; i < 16; ++i) o[q][i] *= k;
          }
        }
#pragma unroll
        for (int q = 0; q < kTiles; ++q)
#pragma unroll
          for (int k = REV ? q : 0; k < (REV ? kTiles : q + 1); ++k) {
            __builtin_amdgcn_sched_barrier(0);
            f32x16 acc = zero16();
#pragma unroll
            for (int x = 0; x < 2 * ND; ++x) {
              uint4 f[L::kPl], own[L::kPl];
              L::load_rows(ta, 32 * q, x, own);
              L::load_rows(tb, 32 * k, x, f);
              acc = dot_planes32(f, own, acc);
            }
            __builtin_amdgcn_sched_barrier(0);
            float z[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int far = 32 * (q - k) + l31 - result_row(i, h), e = REV ? -far : far;
              z[i] = acc[i] * (scale * power[e]);
              if (q == k) z[i] = e >= 0 ? z[i] : 0.f;  // (not finite times 0 is no zero)
            }
            uint4 w[2][L::kPl];
            to_planes<L::kPl>(z, w);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              uint4 f[L::kPl];
#pragma unroll
              for (int i = 0; i < L::kPl; ++i) f[i] = wf[2 * k + x][i];
              if (k == q) {  // (not finite times a masked 0 is no zero)
                const uint4 b = not_finite_entries(f[0]);
#pragma unroll
                for (int i = 0; i < L::kPl; ++i) f[i].x &= ~b.x, f[i].y &= ~b.y, f[i].z &= ~b.z, f[i].w &= ~b.w;
              }
              o[q] = dot_planes32(f, w[x], o[q]);
            }
          }
        if (__builtin_expect(__ballot(bad != 0) != 0, 0)) {
          // values that are not finite, left out of the own tiles: as in contract32_own
          settle_mfma32();
#pragma unroll
          for (int q = 0; q < kTiles; ++q) {
            f32x16 count = zero16();
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              float y[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const int row = result_row(8 * x + i, h);
                y[i] = (REV ? row >= l31 : row <= l31) ? 1.f : 0.f;
              }
              const uint4 b = not_finite_entries(wf[2 * q + x][0]);
              count = mfma32(uint4{b.x & 0x3f803f80u, b.y & 0x3f803f80u, b.z & 0x3f803f80u, b.w & 0x3f803f80u}, to_bf16(y),
                             count);
            }
            settle_mfma32();
#pragma unroll
            for (int i = 0; i < 16; ++i) o[q][i] = count[i] > 0.f ? __uint_as_float(0x7fc00000u) : o[q][i];
          }
        }
        if (!REV || closes) {
          settle_mfma32();
#pragma unroll
          for (int q = 0; q < kTiles; ++q) {
            const int r = 32 * q + l31;
            if (r >= m) continue;
            T* const out = (T*)s.out + (((int64_t)head * (REV ? 1 : s.G) + (REV ? 0 : member)) * s.n + t0 + r) * s.dw;
            const f32x16 one[1] = {o[q]};
            store_row32<T, 1>(out + 32 * wave, s.dw - 32 * wave, one, 1.f, false);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (REV ? opens : closes) {
        const float hi = m == C ? whole.hi : tail.hi, lo = m == C ? whole.lo : tail.lo;
#pragma unroll
        for (int j = 0; j < ND; ++j)
#pragma unroll
          for (int i = 0; i < 16; ++i) S[j][i] = times(S[j][i], FloatPair{hi, lo});
      }
      if (REV || closes) {
#pragma unroll
        for (int x = 0; x < C / 16; ++x) {
          __builtin_amdgcn_sched_barrier(0);
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = 0.f;
#pragma unroll
          for (int i = L::kPl - 1; i >= 0; --i) {
            const uint32_t u4[4] = {wf[x][i].x, wf[x][i].y, wf[x][i].z, wf[x][i].w};
#pragma unroll
            for (int y = 0; y < 4; ++y) v[2 * y] += lo_f32(u4[y]), v[2 * y + 1] += hi_f32(u4[y]);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int r = 16 * x + result_row(i, h);
            v[i] *= s.update * (REV ? early(r) : late(r));
          }
          uint4 w3[1][3];
          to_planes<3>(v, w3);
#pragma unroll
          for (int j = 0; j < ND; ++j) {
            uint4 f[L::kPl];
            L::load_transposed(tb, 16 * x, j, f);
            S[j] = dot_planes32(f, w3[0], S[j]);
          }
        }
        settle_mfma32();
      }
    }
  }
  float* const to = SUMS ? p.states + ((int64_t)head * p.parts + part) * size
                         : !p.states && s.S_out ? s.S_out + head * size : nullptr;
  if (to) {
#pragma unroll
    for (int j = 0; j < ND; ++j)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (has(j, i)) to[state_at(j, i, !p.states && s.transposed)] = S[j][i];
  }
  if (!SUMS && s.out) {
    const int pad = last - end;  // rows behind the sequence
    for (int g = 0; g < (REV ? 1 : s.G); ++g) {
      T* const out = (T*)s.out + (((int64_t)head * (REV ? 1 : s.G) + g) * s.n + end) * s.dw;
      for (int64_t i = tid; i < (int64_t)pad * s.dw; i += kThreads) out[i] = (T)0;
    }
  }
}

// What each part adds becomes what it starts from; one thread per entry of a state.
__global__ void __launch_bounds__(256) decay_carry_kernel(DecayScan s, ScanParts p) {
  const int head = blockIdx.y;
  const int64_t size = (int64_t)s.da * s.dw;
  const int i = blockIdx.x * 256 + threadIdx.x;
  const int len = tokens_of(s.lengths, head / s.H, s.n);
  const float g = s.log_decay[head % s.H];
  const FloatPair whole = decay_power(g, p.part_len);
  if (i >= size) return;
  const int row = i / s.dw, at = s.transposed ? (i - row * s.dw) * s.da + row : i;
  float* const states = p.states + (int64_t)head * p.parts * size + i;
  float R = s.S_in ? s.S_in[head * size + at] : 0.f;
  for (int c = 0; c < p.parts; ++c) {
    const int part = s.reverse ? p.parts - 1 - c : c;
    const int tokens = min(max(len - part * p.part_len, 0), p.part_len);
    const float add = states[part * size];
    states[part * size] = R;
    R = times(R, tokens == p.part_len ? whole : decay_power(g, tokens)) + add;
  }
  if (s.S_out) s.S_out[head * size + at] = R;
}

template <typename T, int ND, bool REV>
hipError_t launch_scan(const DecayScan& s, float* states, hipStream_t st) {
  constexpr int bytes = 3 * PairTile<T, ND, kChunk>::kBytes + 4 * (2 * kChunk + 4);
  static_assert(bytes <= 160 * 1024, "LDS of one workgroup");
  auto scan = decay_scan_kernel<T, ND, REV, false>;
  auto sums = decay_scan_kernel<T, ND, REV, true>;
  if (bytes > 64 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)scan, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) e = hipFuncSetAttribute((const void*)sums, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  ScanParts p{1, s.n, nullptr};
  const DecayScanPlan plan = plan_decay_scan(s.heads, s.n, s.da, s.dw);
  if (plan.parts > 1) {
    p = ScanParts{plan.parts, plan.part_len, states};
    hipLaunchKernelGGL(sums, dim3(s.heads * p.parts), dim3(64 * ND), bytes, st, s, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(decay_carry_kernel, dim3((s.da * s.dw + 255) / 256, s.heads), dim3(256), 0, st, s, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  hipLaunchKernelGGL(scan, dim3(s.heads * p.parts), dim3(64 * ND), bytes, st, s, p);
  return hipGetLastError();
}

template <int ND>
hipError_t launch_scan_n(const DecayScan& s, bool bf16, float* states, hipStream_t st) {
  if (s.reverse) return bf16 ? launch_scan<u16, ND, true>(s, states, st) : launch_scan<float, ND, true>(s, states, st);
  return bf16 ? launch_scan<u16, ND, false>(s, states, st) : launch_scan<float, ND, false>(s, states, st);
}

}  // namespace

DecayScanPlan plan_decay_scan(int heads, int n, int da, int dw) {
  const int tiles = (std::max(da, dw) + 31) / 32;
  DecayScanPlan p;
  const int64_t want = std::max<int64_t>(1, 2048 / tiles / heads);  // (8 waves on each of 256 compute units)
  const int chunks = (n + kChunk - 1) / kChunk;
  const int each = (int)std::max<int64_t>(1, (chunks + want - 1) / want);
  p.parts = std::max(1, (chunks + each - 1) / each);
  p.part_len = each * kChunk;
  p.state_bytes = p.parts > 1 ? sizeof(float) * (size_t)heads * p.parts * da * dw : 0;
  return p;
}

hipError_t launch_decay_scan(const DecayScan& s, bool bf16, float* states, hipStream_t st) {
  switch ((std::max(s.da, s.dw) + 31) / 32) {
    case 1: return launch_scan_n<1>(s, bf16, states, st);
    case 2: return launch_scan_n<2>(s, bf16, states, st);
    case 3: return launch_scan_n<3>(s, bf16, states, st);
    default: return launch_scan_n<4>(s, bf16, states, st);
  }
}

}  // namespace sata
