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

// A workgroup of ND waves takes a part of one head's tokens, in chunks of 32: wave j has the
// state's (and the output's) columns 32 j .. +31 in registers, one in each lane pair.  With r a row
// of a chunk of m tokens and R the state before it (forward)
//     out_r = readout lam^(r+1) a_r R + sum_{s<=r} update readout lam^(r-s) (a_r.b_s) w_s
//     R     = lam^m R + sum_s update lam^(m-1-s) b_s (x) w_s
// and in reverse the same with lam^(m-1-r), lam^(s-r) and lam^(s+1).
//
// Bound: memory (a, b, w read and out written once) is the floor; what it runs at is the chain of a chunk, in
// a wave 16 + 8 + 4 + 24 matrix instructions at d = 128 in bfloat16, some 510 vector instructions
// and two barriers, with two waves a SIMD.  B = 8, H = 16, n = 8192, d = 128 in bfloat16: 468 us
// (2.33 TB/s of 4.9), 0.3 of it the sums; gradients of B = 8, H = 32, n = 2048, d = 64: 210 us
// (2.24 TB/s).  Short prompts and few heads: a part's chunks one after the other, and the launches of the
// sums and the carry.
//
// The state lies in units of f = lam^(tokens since ...): lam^m goes into f, which enters the readout's
// factor and, inverted, the update's; only when f falls below 2^-8 are all entries
// multiplied (not 16 ND products at every chunk).
//
// Precision: bfloat16 inputs are exact operands.  The pairs' weights inside a chunk and the state's entries
// in their readout are two bfloat16 numbers, 2^-17 of them off, for the sums have terms of both signs, which may
// cancel (with one number for the state's entries outputs were 0.0023 off the exact ones, relative,
// instead of 0.0017, the rounding of the output, and the calls above took 9% less: 437 us where these took
// 481, 192 where 213); what is
// added to the state carries 24 bits (w times its power as three), so that the state is a
// float32 one.  float32 inputs, weights and states: three bfloat16 numbers each.
constexpr int kChunk = 32;

// Parts of a head's sequence side by side: states[head][part], as [d_k][d_v], is what each adds to the
// state (written by the sums) and then what it starts from.
struct ScanParts {
  int parts, part_len;  // (tokens: a multiple of the chunk)
  float* states;
};
struct ScanJob {
  DecayScan s;
  ScanParts p;
};
struct ScanJobs {
  ScanJob job[3];
  int jobs;
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

template <typename T, int ND>
struct ScanLds {
  using L = PairTile<T, ND, kChunk>;
  static constexpr int kPowers = 3 * L::kElems;  // (u16 before them)
  static constexpr int kBytes = 2 * kPowers + 4 * (4 * kChunk + 8);
};

// REV: from the last token back.  The members of a group (G) vary in a forward, and in b
// and w in reverse.  SUMS: only what the part adds to the state, from zero.
template <typename T, int ND, bool REV, bool SUMS>
__device__ __forceinline__ void scan_part(const DecayScan& s, const ScanParts& p, int head, int part, u16* smem) {
  constexpr int C = kChunk, kThreads = 64 * ND;
  using D = ScanLds<T, ND>;
  using L = typename D::L;
  constexpr int PS = sizeof(T) == 2 ? 2 : 3;  // numbers of a state's entry in its readout
  constexpr int PA = PS;                      // of a pair's weight
  u16* const ta = smem;
  u16* const tb = smem + L::kElems;
  u16* const tw = tb + L::kElems;
  // Powers of lam at C + exponent, zeros below, and the same times the scale of the scores.  An exponent
  // is a lane's number (at least -4) plus a constant: the lanes' pointers start 4 further
  // on, so that the constants are the instructions' offsets (they took an address register each).
  float* const power = (float*)(smem + D::kPowers);
  float* const scaled = power + 2 * C + 4;
  const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = tokens_of(s.lengths, head / s.H, s.n);
  const int first = part * p.part_len, last = min(first + p.part_len, s.n), end = max(first, min(last, len));
  const int chunks = (end - first + C - 1) / C;
  const int col = 32 * wave + l31;
  const double rate = decay_rate(s.log_decay[head % s.H]);
  for (int e = tid; e <= C; e += kThreads) {
    const float x = (float)decay_power(rate, e);
    power[C + e] = x;
    scaled[C + e] = x * (s.update * s.readout);
    if (e < C) power[e] = scaled[e] = 0.f;
  }

  f32x16 S[ND];
  auto state_at = [&](int j, int i) {
    const int r = 32 * j + result_row(i, h);
    return s.transposed ? (int64_t)col * s.da + r : (int64_t)r * s.dw + col;
  };
  auto has = [&](int j, int i) { return 32 * j + result_row(i, h) < s.da && col < s.dw; };
  const int64_t size = (int64_t)s.da * s.dw;
  float* const states = p.parts > 1 ? p.states + ((int64_t)head * p.parts + part) * size : nullptr;
  const float* const from = SUMS ? nullptr : states ? states : s.S_in ? s.S_in + head * size : nullptr;
#pragma unroll
  for (int j = 0; j < ND; ++j)
#pragma unroll
    for (int i = 0; i < 16; ++i) S[j][i] = from && has(j, i) ? from[state_at(j, i)] : 0.f;
  double f = 1.0, inv = 1.0;  // the state is f S; 1 / f

  if (chunks > 0) {
    const int G = SUMS && !REV ? 1 : s.G, units = chunks * G;
    // (only the chunk at the sequence's end has fewer tokens)
    const int rest = end - first - (chunks - 1) * C;
    const double lam_c = exp(rate * C), lam_r = exp(rate * rest), inv_c = exp(-rate * C), inv_r = exp(-rate * rest);
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
    fetch(0, row_of(0));
    f32x16 o;
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

      // of the rows result_row(i, h) of a chunk's 32 (i a constant)
      const float* const early = power + 4 * h;
      const float* const late = power + m - 1 + 4 - 4 * h;
      auto early_of = [&](int i) { return early[C + 1 + result_row(i, 0)]; };
      auto late_of = [&](int i) { return late[C - 4 - result_row(i, 0)]; };
      // this wave's columns of w: operands of rows 16 x .. +15
      uint4 wf[C / 16][L::kPl];
      uint32_t bad = 0;
#pragma unroll
      for (int x = 0; x < C / 16; ++x) {
        L::load_transposed(tw, 16 * x, wave, wf[x]);
        bad |= not_finite_bits(wf[x][L::kPl - 1]);
      }
      if constexpr (!SUMS) {
        if (!REV || opens) {
          o = zero16();
#pragma unroll
          for (int x = 0; x < 2 * ND; ++x) {
            float v[8];
            uint4 st[1][PS], e[L::kPl];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = S[x / 2][8 * (x & 1) + i];
            to_planes<PS>(v, st);
            load_rows_as_results<L>(ta, 0, x, e);
            o = dot_planes32(st[0], e, o);
          }
          const float k = s.readout * (float)f * (REV ? power[C + m - 1 - l31] : power[C + 1 + l31]);
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] *= k;
        }
        __builtin_amdgcn_sched_barrier(0);
        f32x16 acc = zero16();
#pragma unroll
        for (int x = 0; x < 2 * ND; ++x) {
          uint4 e[L::kPl], own[L::kPl];
          L::load_rows(ta, 0, x, own);
          L::load_rows(tb, 0, x, e);
          acc = dot_planes32(e, own, acc);
        }
        __builtin_amdgcn_sched_barrier(0);
        const float* const ahead = scaled + l31 + 4 - 4 * h;
        const float* const behind = scaled + 32 + 4 * h - l31;
        float z[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const bool sees = REV ? result_row(i, h) >= l31 : result_row(i, h) <= l31;
          float x = REV ? behind[C - 32 + result_row(i, 0)] : ahead[C - 4 - result_row(i, 0)];
          asm volatile("" : "+v"(x));  // (read by all lanes, not in 16 branches)
          z[i] = sees ? acc[i] * x : 0.f;  // (a select: not finite times 0 is no zero)
        }
        if (REV && m < C) {  // (nor are rows behind the sequence, which are zeros, if the decay is not finite)
          stay_in_branch();
#pragma unroll
          for (int i = 0; i < 16; ++i) z[i] = result_row(i, h) < m ? z[i] : 0.f;
        }
        uint4 w[2][PA];
        to_planes<PA>(z, w);
        uint4 wc[2][L::kPl];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int i = 0; i < L::kPl; ++i) wc[x][i] = wf[x][i];
        const bool odd = __ballot(bad != 0) != 0;
        if (__builtin_expect(odd, 0)) {
          // Values of w that are not finite are left out: weights of pairs that are masked are zero, and
          // the product would not be.
          stay_in_branch();
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint4 b = not_finite_entries(wf[x][L::kPl - 1]);
#pragma unroll
            for (int i = 0; i < L::kPl; ++i) wc[x][i].x &= ~b.x, wc[x][i].y &= ~b.y, wc[x][i].z &= ~b.z, wc[x][i].w &= ~b.w;
          }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) o = dot_planes32(wc[x], w[x], o);
        if (__builtin_expect(odd, 0)) {
          // They get their due here: a product of marks with the pairs that are not masked tells which
          // outputs have one, and those are NaN.
          settle_mfma32();
          f32x16 count = zero16();
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int row = result_row(8 * x + i, h);
              y[i] = (REV ? row >= l31 : row <= l31) ? 1.f : 0.f;
            }
            const uint4 b = not_finite_entries(wf[x][L::kPl - 1]);
            count = mfma32(uint4{b.x & 0x3f803f80u, b.y & 0x3f803f80u, b.z & 0x3f803f80u, b.w & 0x3f803f80u}, to_bf16(y),
                           count);
          }
          settle_mfma32();
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] = count[i] > 0.f ? __uint_as_float(0x7fc00000u) : o[i];
        }
        if (!REV || closes) {
          settle_mfma32();
          if (l31 < m) {
            T* const out = (T*)s.out + (((int64_t)head * (REV ? 1 : s.G) + (REV ? 0 : member)) * s.n + t0 + l31) * s.dw;
            const f32x16 one[1] = {o};
            store_row32<T, 1>(out + 32 * wave, s.dw - 32 * wave, one, 1.f, false);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (REV ? opens : closes) {
        f *= m == C ? lam_c : lam_r;
        inv *= m == C ? inv_c : inv_r;
        if (f < 0x1p-8) {
          const float k = (float)f;
#pragma unroll
          for (int j = 0; j < ND; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) S[j][i] *= k;
          f = inv = 1.0;
        }
      }
      if (REV || closes) {
        const float up = s.update * (float)inv;
#pragma unroll
        for (int x = 0; x < C / 16; ++x) {
          __builtin_amdgcn_sched_barrier(0);
          float v[8];
#pragma unroll
          for (int i = L::kPl - 1; i >= 0; --i) {
            const uint32_t u4[4] = {wf[x][i].x, wf[x][i].y, wf[x][i].z, wf[x][i].w};
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              v[2 * y] = i == L::kPl - 1 ? lo_f32(u4[y]) : v[2 * y] + lo_f32(u4[y]);
              v[2 * y + 1] = i == L::kPl - 1 ? hi_f32(u4[y]) : v[2 * y + 1] + hi_f32(u4[y]);
            }
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            v[i] *= up * (REV ? early_of(8 * x + i) : late_of(8 * x + i));
          }
          uint4 w3[1][3];
          to_planes<3>(v, w3);
#pragma unroll
          for (int j = 0; j < ND; ++j) {
            uint4 e[L::kPl];
            L::load_transposed(tb, 16 * x, j, e);
            S[j] = dot_planes32(e, w3[0], S[j]);
          }
        }
        settle_mfma32();
      }
    }
  }
  float* const to = SUMS ? states
                         : s.S_out && part == (REV ? 0 : p.parts - 1) ? s.S_out + head * size : nullptr;
  if (to) {
    const float k = (float)f;
#pragma unroll
    for (int j = 0; j < ND; ++j)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (has(j, i)) to[state_at(j, i)] = S[j][i] * k;
  }
  if (!SUMS) {
    for (int g = 0; g < (REV ? 1 : s.G); ++g) {  // rows behind the sequence
      T* const out = (T*)s.out + (((int64_t)head * (REV ? 1 : s.G) + g) * s.n + end) * s.dw;
      for (int i = tid; i < (last - end) * s.dw; i += kThreads) out[i] = (T)0;
    }
  }
}

template <typename T, int ND, bool SUMS>
__global__ void __launch_bounds__(64 * ND, sizeof(T) == 2 ? 2 : 1) decay_scan_kernel(ScanJobs a) {
  extern __shared__ __attribute__((aligned(16))) u16 smem16[];
  const DecayScan& s0 = a.job[0].s;
  // An XCD takes whole heads: what the jobs and parts of a head read is read through one L2.
  // (nobody reads what the last part adds, in reverse the first)
  const int parts = a.job[0].p.parts - (SUMS ? 1 : 0), each = a.jobs * parts;
  int head, unit;
  if (s0.heads >= 8) {
    const int j = blockIdx.x >> 3;
    head = j / each * 8 + (int)(blockIdx.x & 7);
    unit = j % each;
    if (head >= s0.heads) return;
  } else {
    head = blockIdx.x / each;
    unit = blockIdx.x % each;
  }
  const int job = unit % a.jobs;
  const DecayScan& s = a.job[job].s;
  const int part = unit / a.jobs + (SUMS && s.reverse ? 1 : 0);
  const ScanParts& p = a.job[job].p;
  if (s.reverse) scan_part<T, ND, true, SUMS>(s, p, head, part, smem16);
  else scan_part<T, ND, false, SUMS>(s, p, head, part, smem16);
}

// What each part adds becomes what it starts from; one thread per entry of a state.
__global__ void __launch_bounds__(256) decay_carry_kernel(ScanJobs a) {
  const DecayScan& s = a.job[blockIdx.z].s;
  const ScanParts& p = a.job[blockIdx.z].p;
  const int head = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
  const int64_t size = (int64_t)s.da * s.dw;
  if (i >= size) return;
  const int len = tokens_of(s.lengths, head / s.H, s.n);
  const double rate = decay_rate(s.log_decay[head % s.H]);
  const FloatPair whole = float_pair(decay_power(rate, p.part_len)), rest = float_pair(decay_power(rate, len % p.part_len));
  float* const states = p.states + (int64_t)head * p.parts * size + i;
  float R = s.S_in ? s.S_in[head * size + i] : 0.f;
  constexpr int kAhead = 8;  // parts read at once
  for (int c0 = 0; c0 < p.parts; c0 += kAhead) {
    float add[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const int part = s.reverse ? p.parts - 1 - c0 - x : c0 + x;
      add[x] = c0 + x + 1 < p.parts ? states[part * size] : 0.f;  // (of the last part: not there, nor needed)
    }
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      if (c0 + x >= p.parts) break;
      const int part = s.reverse ? p.parts - 1 - c0 - x : c0 + x, tokens = len - part * p.part_len;
      states[part * size] = R;
      if (tokens >= p.part_len) R = times(R, whole) + add[x];
      else if (tokens > 0) R = times(R, rest) + add[x];
    }
  }
}

template <typename T, int ND, bool SUMS>
hipError_t launch_jobs(const ScanJobs& a, hipStream_t st) {
  constexpr int bytes = ScanLds<T, ND>::kBytes;
  static_assert(bytes <= 160 * 1024, "LDS of one workgroup");
  auto kern = decay_scan_kernel<T, ND, SUMS>;
  if (bytes > 64 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  const int heads = a.job[0].s.heads;
  const int64_t grid = (int64_t)(heads >= 8 ? (heads + 7) / 8 * 8 : heads) * a.jobs * (a.job[0].p.parts - (SUMS ? 1 : 0));
  hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(64 * ND), bytes, st, a);
  return hipGetLastError();
}

template <typename T, int ND>
hipError_t launch_scan(const DecayScan* scans, int count, const DecayScan* sums, int sum_count, float* states,
                       const DecayScanPlan& plan, hipStream_t st) {
  const int64_t size = (int64_t)scans[0].da * scans[0].dw;
  ScanJobs a{};
  if (plan.parts > 1) {
    a.jobs = sum_count;
    for (int i = 0; i < sum_count; ++i)
      a.job[i] = ScanJob{sums[i], {plan.parts, plan.part_len, states + i * scans[0].heads * plan.parts * size}};
    hipError_t e = launch_jobs<T, ND, true>(a, st);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(decay_carry_kernel, dim3((unsigned)((size + 255) / 256), scans[0].heads, sum_count), dim3(256), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  a.jobs = count;
  for (int i = 0; i < count; ++i)
    a.job[i] = ScanJob{scans[i], {plan.parts, plan.part_len,
                                  plan.parts > 1 ? states + (scans[i].reverse ? sum_count - 1 : 0) * scans[0].heads * plan.parts * size
                                                 : nullptr}};
  return launch_jobs<T, ND, false>(a, st);
}

template <int ND>
hipError_t launch_scan_t(const DecayScan* scans, int count, const DecayScan* sums, int sum_count, bool bf16, float* states,
                         const DecayScanPlan& plan, hipStream_t st) {
  return bf16 ? launch_scan<u16, ND>(scans, count, sums, sum_count, states, plan, st)
              : launch_scan<float, ND>(scans, count, sums, sum_count, states, plan, st);
}

}  // namespace

// The number of parts with the least estimated time, in us on an MI355X: chunks one after the other
// in a workgroup, workgroups side by side as far as there are slots (8 waves a compute unit, float32 4), the sums at
// 0.45 of a scan's chunk or the time of their bytes, two launches more and the states read and written.
DecayScanPlan plan_decay_scan(bool bf16, int heads, int G, int n, int da, int dw, int jobs) {
  const int tiles = (std::max(da, dw) + 31) / 32, chunks = std::max(1, (n + kChunk - 1) / kChunk);
  const double unit = bf16 ? 1.6 + 0.6 * tiles : 2.0 + 1.3 * tiles, slots = (bf16 ? 2048.0 : 1024.0) / tiles;
  const int sums = jobs > 1 ? 2 : 1;
  const double bytes = (double)heads * n * (da + dw) * (bf16 ? 2 : 4) * (sums > 1 ? 0.5 * (1 + G) : 1.0);
  DecayScanPlan best;
  double least = 0.0;
  for (int each = chunks; each >= 1; each = each > 8 ? (each + 1) / 2 : each - 1) {
    const int parts = (chunks + each - 1) / each;
    const double wgs = (double)heads * jobs * parts;
    double t = std::max(1.0, wgs / slots) * each * G * unit;
    if (parts > 1) {
      const double work = std::max(1.0, (double)heads * sums * (parts - 1) / slots) * each * (sums > 1 ? 0.5 * (1 + G) : 1.0);
      t += 10.0 + std::max(0.45 * unit * work, bytes * (parts - 1) / parts / 4.5e6) +
           16.0 * sums * heads * parts * da * dw / 4.5e6;
    }
    if (best.part_len == 0 || t < least) {
      least = t;
      best.parts = parts;
      best.part_len = each * kChunk;
    }
    if (each == 1) break;
  }
  best.state_bytes = best.parts > 1 ? sizeof(float) * (size_t)heads * best.parts * da * dw : 0;
  return best;
}

hipError_t launch_decay_scan(const DecayScan* scans, int count, const DecayScan* sums, int sum_count, bool bf16,
                             float* states, hipStream_t st) {
  const DecayScan& s = scans[0];
  const DecayScanPlan plan = plan_decay_scan(bf16, s.heads, s.G, s.n, s.da, s.dw, count);
  switch ((std::max(s.da, s.dw) + 31) / 32) {
    case 1: return launch_scan_t<1>(scans, count, sums, sum_count, bf16, states, plan, st);
    case 2: return launch_scan_t<2>(scans, count, sums, sum_count, bf16, states, plan, st);
    case 3: return launch_scan_t<3>(scans, count, sums, sum_count, bf16, states, plan, st);
    default: return launch_scan_t<4>(scans, count, sums, sum_count, bf16, states, plan, st);
  }
}

}  // namespace sata
