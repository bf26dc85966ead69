// Gradients of the gated delta rule, in four passes: what the blocks' pairs leave (delta_pairs.hip), forward for the
// states before every 64 tokens and the errors E = v - k S' (delta_scan.hpp), backward for the states' gradients U
// and z = dL/du, in the same launch, and then, all blocks of 64 tokens side by side, what a block's tokens
// make of these.  With the letters of delta_tiles.hpp, D = -beta z, S the state before a block and U the gradient behind it:
//     du  = P^T dy + exp(G_C - G) (k U),   P_ij = c exp(G_i - G_j) q_i.k_j (j <= i)
//     z   = (I + M)^-T du,   M_ij = exp(G_i - G_j) beta_i k_i.k_j (j < i),   dv = beta z,   dbeta = z.E
//     U   = exp(G_C) U + (c exp(G) q)^T dy + (exp(G) k)^T D
//     dq  = c exp(G) dy S^T + one k,                 one_ij = c exp(G_i - G_j) dy_i.u_j (j <= i)
//     dk  = asked + kept,  asked = exp(G) D S^T + two k,   two_ij = exp(G_i - G_j) D_i.u_j (j < i)
//                          kept  = one^T q + two^T k + exp(G_C - G) u U^T
//     dg_t = sum_{i>=t} (q.dq + k.asked - k.kept)_i + <U, S behind the block>:
// every term that grows with G_i counts for it, every one that falls against it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "delta_scan.hpp"
#include "delta_tiles.hpp"

namespace sata {

namespace {

constexpr int kBlock = kDeltaBlock;
constexpr int kBackWaves = 4, kBackThreads = 64 * kBackWaves;

// ---- from the last token back: a wave has 16 columns of U, as the forward scan of S, and four more bring blocks into LDS
constexpr int kBackScanThreads = 2 * kBackThreads;
template <typename T, int ND>
struct BackLds {
  using L = DeltaTile<T, ND, kBlock>;
  using Y = SliceStage<T, kBackThreads>;
  static constexpr int kBuffers = sizeof(T) == 2 ? 2 : 1;
  static constexpr int kBuffer = 2 * L::kBytes + (int)sizeof(DeltaBackward) + Y::kBytes;
  static constexpr int kBytes = kBuffers * kBuffer;
  static_assert(kBytes <= 160 * 1024 && kBuffer % 16 == 0, "LDS of one workgroup");
};

template <typename T, int ND>
__device__ __forceinline__ void delta_back(const DeltaArgs& a, const void* data_, float* behind, float* zs, int workgroup, int slices,
                                           u16* smem16) {
  using D = BackLds<T, ND>;
  using L = typename D::L;
  using Data = DeltaBackward;
  using Y = typename D::Y;
  int head, slice;
  if (!delta_place(workgroup, a.heads, slices, head, slice)) return;
  const int tid = threadIdx.x, lane = tid & 63, l15 = lane & 15, t4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t shared = head / a.G;
  const int len = tokens_of(a.lengths, head / (a.Hk * a.G), a.n), blocks = (len + kBlock - 1) / kBlock;
  const int64_t all_blocks = (a.n + kBlock - 1) / kBlock, head0 = (int64_t)head * a.n * a.dv;
  auto buffer = [&](int c) { return smem16 + (D::kBuffers == 2 && (c & 1) ? D::kBuffer / 2 : 0); };
  if (wave >= kBackWaves) {  // ---- the next block into LDS
    const int id = tid - kBackThreads;
    DeltaStage<T, ND, kBlock, kBackThreads> sq, sk;
    DataStage<Data, kBackThreads> sd;
    Y sy;
    sq.init((const T*)a.q + shared * a.n * a.dk, len, a.dk, id);
    sk.init((const T*)a.k + shared * a.n * a.dk, len, a.dk, id);
    sd.init((const Data*)data_ + head * all_blocks, blocks, id);
    sy.init((const T*)a.dy + head0, len, a.dv, 64 * slice, id);
    auto fetch = [&](int c) {
      sk.fetch(c * kBlock);
      sq.fetch(c * kBlock);
      sd.fetch(c);
      sy.fetch(c * kBlock);
    };
    if (blocks > 0) fetch(blocks - 1);
    for (int c = blocks - 1; c >= 0; --c) {
      u16* const tk = buffer(c);
      if (D::kBuffers == 1 && c + 1 < blocks) __syncthreads();  // (the block behind has been read)
      sk.put(tk, c * kBlock);
      sq.put(tk + L::kElems, c * kBlock);
      sd.put((Data*)(tk + 2 * L::kElems));
      sy.put((T*)((Data*)(tk + 2 * L::kElems) + 1), c * kBlock);
      __syncthreads();
      if (c > 0) fetch(c - 1);
    }
    return;
  }
  const int col = 16 * (kBackWaves * slice + wave) + l15;
  const bool on = col < a.dv;
  const int64_t size = (int64_t)a.dk * a.dv;
  f32x4 U[2 * ND];
#pragma unroll
  for (int j = 0; j < 2 * ND; ++j) U[j] = zero4();
  StateColumns state;
  if (a.dS) {
    state.init(a.dS + head * size, a.dk, a.dv, col);
    state.load(U);
  }
  {
    ColumnStage<T> sv;
    ColumnStage<float> sz;
    sv.init((const T*)a.dv_out + head0, len, a.dv, col);
    sz.init(zs + head0, len, a.dv, col);
    for (int c = blocks - 1; c >= 0; --c) {
      const int t0 = c * kBlock;
      const u16* const tk = buffer(c);
      const u16* const tq = tk + L::kElems;
      const Data& d = *(const Data*)(tq + L::kElems);
      if (D::kBuffers == 1 && c + 1 < blocks) __syncthreads();
      __syncthreads();
      const T* const ys = (const T*)(&d + 1) + 16 * wave + l15;
      float y[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] = entry_of(ys, (16 * (e >> 2) + 4 * t4 + (e & 3)) * Y::kPitch);
      state.init(behind + (head * all_blocks + c) * size, a.dk, a.dv, col);
      state.store(U);
      auto operand = [&](const DeltaOperand* p, int x, uint4 (&op)[3]) {
#pragma unroll
        for (int i = 0; i < 3; ++i) op[i] = p[i][x][lane];
      };
      f32x4 early[4], late[4], beta[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        early[x] = *(const f32x4*)(d.early + 16 * x + 4 * t4);
        late[x] = *(const f32x4*)(d.late + 16 * x + 4 * t4);
        beta[x] = *(const f32x4*)(d.beta + 16 * x + 4 * t4);
      }
      const FloatPair whole = d.whole;
      f32x4 R[4] = {zero4(), zero4(), zero4(), zero4()}, z[4];
#pragma unroll
      for (int b = 0; b < ND; ++b) {
        uint4 st[3], e[4][L::kPl];
        operand_of<3>(U[2 * b], U[2 * b + 1], st);
#pragma unroll
        for (int x = 0; x < 4; ++x) rows16<L>(tk, 16 * x, b, e[x]);
        dots_left16(e, st, R);
      }
      uint4 yp[2][L::kPl], ep[2][3], zp[3], wp[2][3];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x8[8], e8[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x8[e] = y[8 * h + e];
          e8[e] = x8[e] * (early[2 * h + (e >> 2)][e & 3] * a.scale);
        }
        operand_of<L::kPl>(x8, yp[h]);
        operand_of<3>(e8, ep[h]);
      }
#pragma unroll
      for (int j = 0; j < 2 * ND; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) U[j][i] = times(U[j][i], whole);
      // the second half first: the first one's updates are seen by its keys
#pragma unroll
      for (int h = 1; h >= 0; --h) {
        f32x4 du[2] = {zero4(), zero4()};
        uint4 p[2][3];
        auto load = [&](const DeltaOperand* from) {
#pragma unroll
          for (int x = 0; x < 2; ++x) operand(from, x, p[x]);
        };
        if (h == 0) {
          load(d.below);
          dots_left16(p, zp, du);
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) du[x][i] = -du[x][i];
          load(d.pairs[1]);
          dots_left16(p, yp[1], du);
        }
        load(d.pairs[2 * h]);
        dots_left16(p, yp[h], du);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i) du[x][i] = fmaf(late[2 * h + x][i], R[2 * h + x][i], du[x][i]);
        uint4 dp[3];
        operand_of<3>(du[0], du[1], dp);
        load(d.inverse[h]);
        f32x4 w[2] = {zero4(), zero4()};
        dots_left16(p, dp, w);
        {  // (between the products that wait for each other)
          uint4 e[2 * ND][L::kPl];
#pragma unroll
          for (int j = 0; j < 2 * ND; ++j) state_columns16<L>(tq, 32 * h, j, e[j]);
          dots_left16(e, ep[h], U);
        }
        z[2 * h] = w[0], z[2 * h + 1] = w[1];
        if (h == 1) operand_of<3>(w[0], w[1], zp);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int x = 2 * h + (e >> 2), i = e & 3;
          w[e] = beta[x][i] * z[x][i];
          sz.store(t0, 8 * h + e, z[x][i]);
          sv.store(t0, 8 * h + e, w[e]);
          w[e] *= -early[x][i];
        }
        operand_of<3>(w, wp[h]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint4 e[2 * ND][L::kPl];
#pragma unroll
        for (int j = 0; j < 2 * ND; ++j) state_columns16<L>(tk, 32 * h, j, e[j]);
        dots_left16(e, wp[h], U);
      }
      settle_mfma();
    }
  }
  if (a.dS_in) {
    state.init(a.dS_in + head * size, a.dk, a.dv, col);
    state.store(U);
  }
  if (on) {
    T* const dv = (T*)a.dv_out + (int64_t)head * a.n * a.dv + col;
    for (int t = len + t4; t < a.n; t += 4) dv[(int64_t)t * a.dv] = (T)0;
  }
}

// Neither scan needs the other: side by side they take little more time than the longer one as long as the card has room.
// 64 heads of 2048 tokens, d_k = d_v = 128, bfloat16: 165 us, one behind the other 144 + 117.
template <typename T, int ND>
__global__ void __launch_bounds__(kBackScanThreads, 2)
delta_scans_kernel(DeltaArgs a, const void* data, const void* back, float* states, float* behind, float* errors, float* zs, int slices) {
  static_assert(kBackScanThreads == kScanThreads, "one launch for both");
  extern __shared__ __attribute__((aligned(16))) u16 smem16[];
  const int half = (int)(gridDim.x / 2), i = (int)blockIdx.x;
  if (i < half) delta_back<T, ND>(a, back, behind, zs, i, slices, smem16);
  else delta_scan<T, ND, true>(a, data, states, errors, i - half, slices, smem16);
}

// ---- block by block: a wave has 16 of 64 tokens and all columns of their dq and dk
//
// float32 calls: first dq and asked, which take what lies before a token (pairs with tokens j <= i, the state before the
// block); then, on top of asked, kept, which takes what lies behind (pairs with i >= j, the gradient of the state behind the
// block).  A pair's weight is formed in both places, once for each side's rows, so that it is an operand where it is formed.
// A block's five tiles of three numbers an entry would take 240 KB of LDS: two lie there at a time.  6 heads x 555
// tokens, d_k = 48, d_v = 32: 24 us, one workgroup's phases behind one another on 108 of the CUs.
template <int ND>
struct BlockLds {
  using L = DeltaTile<float, ND, kBlock>;  // errors, z, gradients of the outputs or rows of a state; queries or keys
  using Half = DeltaTile<float, ND, 32>;
  static constexpr int kBytes = 2 * L::kBytes;
};

// Sums over the lanes up to (or from) a lane's own.
__device__ __forceinline__ double sum_up_to(double x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __shfl_up((uint32_t)u, d), hi = __shfl_up((uint32_t)(u >> 32), d);
    if (lane >= d) x += __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
  }
  return x;
}
__device__ __forceinline__ double sum_from(double x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __shfl_down((uint32_t)u, d), hi = __shfl_down((uint32_t)(u >> 32), d);
    if (lane + d < 64) x += __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
  }
  return x;
}

// A lane's entry of a staged tile, of row r0 + 4 t4 + r and column 16 j + l15.
template <typename L>
__device__ __forceinline__ float tile_entry(const u16* t, int row, int col) {
  const u16* const p = t + L::at(row, col);
  float x = __uint_as_float((uint32_t)p[0] << 16);
#pragma unroll
  for (int i = 1; i < L::kPl; ++i) x += __uint_as_float((uint32_t)p[i * L::kPlane] << 16);
  return x;
}

// Lanes to a row of by_rows.
template <int ND>
constexpr int by_rows_lanes() { return ND == 1 ? 4 : ND == 2 ? 8 : 16; }

// A wave's results of 16 tokens by 32 ND columns, through LDS into rows: row(i, c0, x) for eight columns at a time.  `buf`: the wave's
// own; 16 rows of 32 ND + 4 floats.  (Results lie by columns: of 16 tokens each lane would write two bytes at a time.)
template <int ND, typename F>
__device__ __forceinline__ void by_rows(const f32x4 (&x)[2 * ND], float* buf, F&& row) {
  constexpr int kPitch = 32 * ND + 4, kLanes = by_rows_lanes<ND>();
  const int lane = threadIdx.x & 63, l15 = lane & 15, t4 = lane >> 4;
  wave_lds_fence();
#pragma unroll
  for (int j = 0; j < 2 * ND; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) buf[(4 * t4 + r) * kPitch + 16 * j + l15] = x[j][r];
  wave_lds_fence();
#pragma unroll
  for (int i = 0; i < kLanes / 4; ++i) {
    const int token = i * (64 / kLanes) + lane / kLanes, c0 = 8 * (lane % kLanes);
    float y[8];
#pragma unroll
    for (int h = 0; h < 8; h += 4) {
      const float4 f = c0 < 32 * ND ? *(const float4*)(buf + token * kPitch + c0 + h) : float4{0.f, 0.f, 0.f, 0.f};
      y[h] = f.x, y[h + 1] = f.y, y[h + 2] = f.z, y[h + 3] = f.w;
    }
    row(token, c0, y);
  }
}

// MANY: several value heads to a query and key head, whose dq and dk are each written to `sums`, [2][value heads][n][dk].
template <int ND, bool MANY>
__global__ void __launch_bounds__(kBackThreads, 1)
delta_blocks_kernel(DeltaArgs a, const float* states, const float* behind, const float* errors, const float* zs, float* sums_) {
  extern __shared__ __attribute__((aligned(16))) u16 smem16[];
  using T = float;
  using D = BlockLds<ND>;
  using L = typename D::L;
  using Half = typename D::Half;
  constexpr int kPl = L::kPl;
  __shared__ double sums[kBlock];
  __shared__ float rates[kBlock], terms[kBlock], parts[kBackWaves];
  u16* const ta = smem16;
  u16* const tb = smem16 + L::kElems;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int blocks = (a.n + kBlock - 1) / kBlock, block = blockIdx.x, head = blockIdx.y, shared = MANY ? head / a.G : head, t0 = block * kBlock;
  const int len = tokens_of(a.lengths, shared / a.Hk, a.n), own = 16 * wave, last = min(a.n, t0 + kBlock);
  const int64_t size = (int64_t)a.dk * a.dv, row0 = (int64_t)shared * a.n, row = (int64_t)head * a.n;
  // rows behind the sequence (several heads' sums: delta_sums_kernel)
  const int rest = max(t0, min(len, last));
  if (!MANY)
    for (int i = tid; i < (last - rest) * a.dk; i += kBackThreads) {
      const int64_t at = (row0 + rest) * a.dk + i;
      ((T*)a.dq)[at] = ((T*)a.dk_out)[at] = (T)0;
    }
  if (tid < kBlock && t0 + tid < last && t0 + tid >= len) a.dg[row + t0 + tid] = a.dbeta[row + t0 + tid] = 0.f;
  if (t0 >= len) return;
  float* const buf = (float*)ta + wave * 16 * (32 * ND + 4);
  static_assert(kBackWaves * 16 * (32 * ND + 4) * 4 <= L::kBytes, "results lie in the errors' place");
  const int l15 = lane & 15, t4 = lane >> 4;
  const T* const q = (const T*)a.q + row0 * a.dk;
  const T* const k = (const T*)a.k + row0 * a.dk;
  const float* const S = states + ((int64_t)head * blocks + block) * size;
  const float* const U = behind + ((int64_t)head * blocks + block) * size;
  RowAccess<float> E, Z;
  RowAccess<T> dy;
  E.init(errors + row * a.dv, len, a.dv);
  Z.init(zs + row * a.dv, len, a.dv);
  dy.init((const T*)a.dy + row * a.dv, len, a.dv);
  DeltaStage<T, ND, kBlock, kBackThreads> sb;
  DeltaStage<float, ND, kBlock, kBackThreads> sa;
  sa.init(errors + row * a.dv, len, a.dv, tid);
  sa.fetch(t0);
  sb.init(k, len, a.dk, tid);
  sb.fetch(t0);
  if (wave == 0) {
    const bool there = t0 + lane < len;
    sums[lane] = sum_up_to(there ? delta_rate(a.g[row + t0 + lane]) : 0.0);
    rates[lane] = there ? a.beta[row + t0 + lane] : 0.f;
  }
  sa.put(ta, t0);
  sb.put(tb, t0);
  __syncthreads();
  const int mine = own + l15;  // a token of this wave's, in the block
  const double my_sum = sums[mine];
  const float my_rate = rates[mine];
  auto decay = [&](double d) { return exp2_fast((float)(d * 1.4426950408889634)); };
  // dots of this wave's tokens' rows, of by_rows: sums over a row's lanes to `terms`
  auto add_term = [&](float x, int token) {
#pragma unroll
    for (int d = 1; d < by_rows_lanes<ND>(); d *= 2) x += __shfl_xor(x, d);
    if (lane % by_rows_lanes<ND>() == 0) terms[own + token] += x;
  };
  // a finished gradient's rows
  auto finish = [&](int which, int token, int c0, float (&x)[8]) {
    RowAccess<std::conditional_t<MANY, float, T>> out;
    if constexpr (MANY) out.init(sums_ + ((int64_t)which * a.heads + head) * a.n * a.dk, len, a.dk);
    else out.init((const T*)(which ? a.dk_out : a.dq) + row0 * a.dk, len, a.dk);
    out.store(t0 + own + token, c0, x);
  };
  float asked_at[4] = {0.f, 0.f, 0.f, 0.f};  // k.asked of tokens own + 4 t4 .. +3, this lane's part
  f32x4 sum_k[2 * ND];
#pragma unroll
  for (int j = 0; j < 2 * ND; ++j) sum_k[j] = zero4();
  {
    f32x4 dq[2 * ND];
#pragma unroll
    for (int j = 0; j < 2 * ND; ++j) dq[j] = zero4();
    uint4 y[ND][kPl], z[ND][3];
#pragma unroll
    for (int s = 0; s < ND; ++s) {
      dy.template operand<kPl>(t0 + mine, 32 * s + 8 * t4, y[s]);
      Z.template operand<3>(t0 + mine, 32 * s + 8 * t4, z[s]);
    }
    // ---- pairs of this wave's tokens i with j <= i: rows of one and two
#pragma unroll 1
    for (int jb = 0; 32 * jb <= own; ++jb) {
      float one[8], two[8];
      f32x4 p[2] = {zero4(), zero4()}, r[2] = {zero4(), zero4()};
#pragma unroll
      for (int s = 0; s < ND; ++s) {
        uint4 e[2][3];
#pragma unroll
        for (int x = 0; x < 2; ++x) rows16<L>(ta, 32 * jb + 16 * x, s, e[x]);
        dots_left16(e, y[s], p);
        dots_left16(e, z[s], r);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int j = 32 * jb + 16 * (e >> 2) + 4 * t4 + (e & 3);
        const float d = decay(my_sum - sums[j]) * rates[j];
        one[e] = j <= mine ? p[e >> 2][e & 3] * d * a.scale : 0.f;
        two[e] = j < mine ? -(r[e >> 2][e & 3] * d * my_rate) : 0.f;
      }
      uint4 op[3], tp[3];
      operand_of<3>(one, op);
      operand_of<3>(two, tp);
#pragma unroll
      for (int j = 0; j < 2 * ND; j += 2) {
        __builtin_amdgcn_sched_barrier(0);
        uint4 e[2][kPl];
        f32x4 w[2] = {dq[j], dq[j + 1]}, u[2] = {sum_k[j], sum_k[j + 1]};
#pragma unroll
        for (int x = 0; x < 2; ++x) columns16<L>(tb, 32 * jb, j + x, e[x]);
        dots_right16(op, e, w);
        dots_right16(tp, e, u);
        dq[j] = w[0], dq[j + 1] = w[1], sum_k[j] = u[0], sum_k[j + 1] = u[1];
      }
      settle_mfma();
    }
    // ---- the state before the block, 32 rows at a time
    float early[4], rate[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) early[r] = decay(sums[own + 4 * t4 + r]), rate[r] = rates[own + 4 * t4 + r];
    DeltaStage<float, ND, 32, kBackThreads> ss;
    ss.init(S, a.dk, a.dv, tid);
    ss.fetch(0);
#pragma unroll
    for (int b = 0; b < ND; ++b)
      if (32 * b < a.dk) {
        __syncthreads();
        ss.put(ta, 32 * b);
        __syncthreads();
        if (32 * b + 32 < a.dk) ss.fetch(32 * b + 32);
        f32x4 of_y[2] = {zero4(), zero4()}, of_z[2] = {zero4(), zero4()};
#pragma unroll
        for (int s = 0; s < ND; ++s) {
          uint4 e[2][3];
#pragma unroll
          for (int x = 0; x < 2; ++x) rows16<Half>(ta, 16 * x, s, e[x]);
          dots_right16(y[s], e, of_y);
          dots_right16(z[s], e, of_z);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            dq[2 * b + x][r] = fmaf(of_y[x][r], early[r] * a.scale, dq[2 * b + x][r]);
            sum_k[2 * b + x][r] = fmaf(-of_z[x][r], early[r] * rate[r], sum_k[2 * b + x][r]);
          }
        settle_mfma();
      }
    // ---- dq is done; asked with the keys
#pragma unroll
    for (int j = 0; j < 2 * ND; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        asked_at[r] = fmaf(tile_entry<L>(tb, own + 4 * t4 + r, 16 * j + l15), sum_k[j][r], asked_at[r]);
    if (lane < 16) terms[own + lane] = 0.f;
    __syncthreads();
    RowAccess<T> rq;
    rq.init(q, len, a.dk);
    by_rows<ND>(dq, buf, [&](int token, int c0, float (&x)[8]) {
      float w[8], dot = 0.f;
      rq.load(t0 + own + token, c0, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) dot = fmaf(w[i], x[i], dot);
      add_term(dot, token);
      finish(0, token, c0, x);
    });
  }
  // ---- pairs of tokens i with this wave's j <= i: columns of one, then of two
  uint4 e_own[ND][3];
  {
    DeltaStage<T, ND, kBlock, kBackThreads> sy;
    sy.init((const T*)a.dy + row * a.dv, len, a.dv, tid);
    sy.fetch(t0);
    sb.init(q, len, a.dk, tid);
    sb.fetch(t0);
    float dot = 0.f;
#pragma unroll
    for (int s = 0; s < ND; ++s) {
      float x[8], w[8];
      E.load(t0 + mine, 32 * s + 8 * t4, x);
      Z.load(t0 + mine, 32 * s + 8 * t4, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) dot = fmaf(x[i], w[i], dot);
      operand_of<3>(x, e_own[s]);
    }
    dot += __shfl_xor(dot, 16);
    dot += __shfl_xor(dot, 32);
    if (t4 == 0 && t0 + mine < len) a.dbeta[row + t0 + mine] = dot;
    __syncthreads();
    sy.put(ta, t0);
    sb.put(tb, t0);
    __syncthreads();
  }
#pragma unroll 1
  for (int turn = 0; turn < 2; ++turn) {
    if (turn == 1) {
      sa.init(zs + row * a.dv, len, a.dv, tid);
      sa.fetch(t0);
      sb.init(k, len, a.dk, tid);
      sb.fetch(t0);
      __syncthreads();
      sa.put(ta, t0);
      sb.put(tb, t0);
      __syncthreads();
    }
#pragma unroll 1
    for (int ib = own / 32; ib < 2; ++ib) {
      float w[8];
      f32x4 p[2] = {zero4(), zero4()};
#pragma unroll
      for (int s = 0; s < ND; ++s) {
        uint4 e[2][3];
#pragma unroll
        for (int x = 0; x < 2; ++x) rows16<L>(ta, 32 * ib + 16 * x, s, e[x]);
        dots_left16(e, e_own[s], p);
      }
      settle_mfma();
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = 32 * ib + 16 * (e >> 2) + 4 * t4 + (e & 3);
        const float d = p[e >> 2][e & 3] * (decay(sums[i] - my_sum) * my_rate);
        w[e] = turn == 0 ? (i >= mine ? d * a.scale : 0.f) : i > mine ? -(d * rates[i]) : 0.f;
      }
      uint4 op[3];
      operand_of<3>(w, op);
#pragma unroll
      for (int j = 0; j < 2 * ND; j += 2) {
        __builtin_amdgcn_sched_barrier(0);
        uint4 e[2][kPl];
        f32x4 u[2] = {sum_k[j], sum_k[j + 1]};
#pragma unroll
        for (int x = 0; x < 2; ++x) columns16<L>(tb, 32 * ib, j + x, e[x]);
        dots_right16(op, e, u);
        sum_k[j] = u[0], sum_k[j + 1] = u[1];
      }
      settle_mfma();
    }
  }
  // ---- the gradient of the state behind the block
  float inner = 0.f, late_terms = 0.f;
  {
    const double end = sums[kBlock - 1];
    float late[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) late[r] = decay(end - sums[own + 4 * t4 + r]) * rates[own + 4 * t4 + r];
    DeltaStage<float, ND, 32, kBackThreads> ss, su;
    ss.init(S, a.dk, a.dv, tid);
    su.init(U, a.dk, a.dv, tid);
    su.fetch(0);
    ss.fetch(0);
#pragma unroll
    for (int b = 0; b < ND; ++b)
      if (32 * b < a.dk) {
        __syncthreads();
        su.put(ta, 32 * b);
        if (su.vec && ss.vec) {
#pragma unroll
          for (int i = 0; i < su.kIt; ++i) {
            inner = fmaf(__uint_as_float(ss.r[i].x), __uint_as_float(su.r[i].x), inner);
            inner = fmaf(__uint_as_float(ss.r[i].y), __uint_as_float(su.r[i].y), inner);
            inner = fmaf(__uint_as_float(ss.r[i].z), __uint_as_float(su.r[i].z), inner);
            inner = fmaf(__uint_as_float(ss.r[i].w), __uint_as_float(su.r[i].w), inner);
          }
        } else {
          for (int i = tid; i < min(32, a.dk - 32 * b) * a.dv; i += kBackThreads)
            inner = fmaf(S[(int64_t)32 * b * a.dv + i], U[(int64_t)32 * b * a.dv + i], inner);
        }
        __syncthreads();
        if (32 * b + 32 < a.dk) {
          su.fetch(32 * b + 32);
          ss.fetch(32 * b + 32);
        }
        f32x4 of_e[2] = {zero4(), zero4()};
#pragma unroll
        for (int s = 0; s < ND; ++s) {
          uint4 e[2][3];
#pragma unroll
          for (int x = 0; x < 2; ++x) rows16<Half>(ta, 16 * x, s, e[x]);
          dots_right16(e_own[s], e, of_e);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float e = of_e[x][r] * late[r];
            late_terms = fmaf(tile_entry<L>(tb, own + 4 * t4 + r, 32 * b + 16 * x + l15), e, late_terms);
            sum_k[2 * b + x][r] += e;
          }
        settle_mfma();
      }
    inner *= decay(end);
  }
  // ---- dk, and the gradient of g (asked counts for it: with kept it has been taken off)
  __syncthreads();
  RowAccess<T> rk;
  rk.init(k, len, a.dk);
  by_rows<ND>(sum_k, buf, [&](int token, int c0, float (&x)[8]) {
    float w[8], dot = 0.f;
    rk.load(t0 + own + token, c0, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) dot = fmaf(w[i], x[i], dot);
    add_term(-dot, token);
    finish(1, token, c0, x);
  });
#pragma unroll
  for (int r = 0; r < 4; ++r) {
#pragma unroll
    for (int d = 1; d < 16; d *= 2) asked_at[r] += __shfl_xor(asked_at[r], d);
    wave_lds_fence();
    if (l15 == r) terms[own + 4 * t4 + r] += 2.f * asked_at[r];
  }
  inner += late_terms;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) inner += __shfl_xor(inner, d);
  if (lane == 0) parts[wave] = inner;
  __syncthreads();
  if (wave == 0) {
    double sum = sum_from(terms[lane]);
#pragma unroll
    for (int w = 0; w < kBackWaves; ++w) sum += parts[w];
    if (t0 + lane < len) a.dg[row + t0 + lane] = (float)sum;
  }
}

// ---- the same for bfloat16 calls, whose tiles of a block lie in LDS together: eight waves, each with 16 tokens and one of the two
// parts.  The first four form dq and asked: pairs with tokens j <= i, the state before the block; the others
// kept: pairs with i >= j, the gradient behind it.  A block's rows are read once, its states once, 32 rows of both at
// a time, and the two parts of dk meet in LDS.  (Of a SIMD's two waves one has the longer part of the pairs, the other
// the shorter.)
// 64 heads x 2048 tokens of 128: 208 us for 557 MB, vector issue 37%, LDS 34%, matrix cores 26% of the cycles; four waves
// that did one part after the other, two workgroups a CU: 320.
template <int ND>
struct SplitLds {
  using W = DeltaTile<float, ND, kBlock>;  // errors, z; later rows of the states
  using L = DeltaTile<u16, ND, kBlock>;    // gradients of the outputs, keys, queries
  using Half = DeltaTile<float, ND, 32>;
  static constexpr int kRows = 16 * (32 * ND + 4);  // floats of a wave's place in by_rows
  static constexpr int kBytes = 2 * W::kBytes + 3 * L::kBytes;
  static_assert(2 * Half::kBytes <= W::kBytes, "rows of both states lie in the errors' place, or z's");
  static_assert(kBackWaves * 2 * ND * 1024 + 2 * kBackWaves * kRows * 4 <= 2 * W::kBytes + L::kBytes, "results lie in front of the keys");
};
constexpr int kSplitThreads = 2 * kBackThreads;

template <int ND, bool MANY>
__global__ void __launch_bounds__(kSplitThreads, 2)
delta_split_kernel(DeltaArgs a, const float* states, const float* behind, const float* errors, const float* zs, float* sums_) {
  extern __shared__ __attribute__((aligned(16))) u16 smem16[];
  using T = u16;
  using D = SplitLds<ND>;
  using W = typename D::W;
  using L = typename D::L;
  using Half = typename D::Half;
  __shared__ double sums[kBlock];
  __shared__ float rates[kBlock], terms[2][kBlock], parts[2 * kBackWaves];
  u16 *const te = smem16, *const tz = te + W::kElems, *const ty = tz + W::kElems, *const tk = ty + L::kElems, *const tq = tk + L::kElems;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), own = 16 * (wave % kBackWaves);
  const bool asks = wave < kBackWaves;
  const int blocks = (a.n + kBlock - 1) / kBlock, block = blockIdx.x, head = blockIdx.y, shared = MANY ? head / a.G : head, t0 = block * kBlock;
  const int len = tokens_of(a.lengths, shared / a.Hk, a.n), last = min(a.n, t0 + kBlock);
  const int64_t size = (int64_t)a.dk * a.dv, row0 = (int64_t)shared * a.n, row = (int64_t)head * a.n;
  // rows behind the sequence (several heads' sums: delta_sums_kernel)
  const int rest = max(t0, min(len, last));
  if (!MANY)
    for (int i = tid; i < (last - rest) * a.dk; i += kSplitThreads) {
      const int64_t at = (row0 + rest) * a.dk + i;
      ((T*)a.dq)[at] = ((T*)a.dk_out)[at] = (T)0;
    }
  if (tid < kBlock && t0 + tid < last && t0 + tid >= len) a.dg[row + t0 + tid] = a.dbeta[row + t0 + tid] = 0.f;
  if (t0 >= len) return;
  const int l15 = lane & 15, t4 = lane >> 4;
  const float* const S = states + ((int64_t)head * blocks + block) * size;
  const float* const U = behind + ((int64_t)head * blocks + block) * size;
  DeltaStage<float, ND, 32, kSplitThreads> ss, su;
  ss.init(S, a.dk, a.dv, tid);
  su.init(U, a.dk, a.dv, tid);
  {
    DeltaStage<float, ND, kBlock, kSplitThreads> se, sz;
    DeltaStage<T, ND, kBlock, kSplitThreads> sy, sk, sq;
    se.init(errors + row * a.dv, len, a.dv, tid);
    se.fetch(t0);
    sy.init((const T*)a.dy + row * a.dv, len, a.dv, tid);
    sy.fetch(t0);
    sz.init(zs + row * a.dv, len, a.dv, tid);
    sz.fetch(t0);
    sk.init((const T*)a.k + row0 * a.dk, len, a.dk, tid);
    sq.init((const T*)a.q + row0 * a.dk, len, a.dk, tid);
    sk.fetch(t0);
    sq.fetch(t0);
    if (wave == 0) {
      const bool there = t0 + lane < len;
      sums[lane] = sum_up_to(there ? delta_rate(a.g[row + t0 + lane]) : 0.0);
      rates[lane] = there ? a.beta[row + t0 + lane] : 0.f;
    }
    se.put(te, t0);
    sy.put(ty, t0);
    sz.put(tz, t0);
    sk.put(tk, t0);
    sq.put(tq, t0);
  }
  ss.fetch(0);
  su.fetch(0);
  __syncthreads();
  const int mine = own + l15;  // a token of this wave's, in the block
  const double my_sum = sums[mine];
  const float my_rate = rates[mine];
  auto decay = [&](double d) { return exp2_fast((float)(d * 1.4426950408889634)); };
  // Rows of the states, 32 at a time, from registers into the errors' and z's places in turn.
  float inner = 0.f;  // this thread's part of <S, U>
  const bool vec = su.vec && ss.vec;
  auto next_rows = [&](int b) {
    u16* const to = b & 1 ? tz : te;
    if (b == 0) __syncthreads();  // (the errors and z have been read)
    ss.put(to, 32 * b);
    su.put(to + Half::kElems, 32 * b);
    if (vec) {
#pragma unroll
      for (int i = 0; i < su.kIt; ++i) {
        inner = fmaf(__uint_as_float(ss.r[i].x), __uint_as_float(su.r[i].x), inner);
        inner = fmaf(__uint_as_float(ss.r[i].y), __uint_as_float(su.r[i].y), inner);
        inner = fmaf(__uint_as_float(ss.r[i].z), __uint_as_float(su.r[i].z), inner);
        inner = fmaf(__uint_as_float(ss.r[i].w), __uint_as_float(su.r[i].w), inner);
      }
    } else {
      for (int i = tid; i < min(32, a.dk - 32 * b) * a.dv; i += kSplitThreads)
        inner = fmaf(S[(int64_t)32 * b * a.dv + i], U[(int64_t)32 * b * a.dv + i], inner);
    }
    __syncthreads();  // (and the rows before the last ones have been read)
    if (32 * b + 32 < a.dk) {
      ss.fetch(32 * b + 32);
      su.fetch(32 * b + 32);
    }
    return to;
  };
  // what a wave's sums over columns add to its tokens' terms
  auto add_terms = [&](float (&x)[4]) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
      for (int d = 1; d < 16; d *= 2) x[r] += __shfl_xor(x[r], d);
      if (l15 == r) terms[asks ? 0 : 1][own + 4 * t4 + r] = x[r];
    }
  };
  f32x4* const meet = (f32x4*)smem16 + own / 16 * 2 * ND * 64;
  float* const buf = (float*)smem16 + kBackWaves * 2 * ND * 256 + wave * D::kRows;
  // a finished gradient's rows
  auto finish = [&](int which, int token, int c0, float (&x)[8]) {
    RowAccess<std::conditional_t<MANY, float, T>> out;
    if constexpr (MANY) out.init(sums_ + ((int64_t)which * a.heads + head) * a.n * a.dk, len, a.dk);
    else out.init((const T*)(which ? a.dk_out : a.dq) + row0 * a.dk, len, a.dk);
    out.store(t0 + own + token, c0, x);
  };
  if (asks) {
    f32x4 dq[2 * ND], asked[2 * ND];
#pragma unroll
    for (int j = 0; j < 2 * ND; ++j) dq[j] = asked[j] = zero4();
    uint4 y[ND][1], z[ND][3];
#pragma unroll
    for (int s = 0; s < ND; ++s) {
      rows16<L>(ty, own, s, y[s]);
      rows16<W>(tz, own, s, z[s]);
    }
#pragma unroll 1
    for (int jb = 0; 32 * jb <= own; ++jb) {
      float one[8], two[8];
      f32x4 p[2] = {zero4(), zero4()}, r[2] = {zero4(), zero4()};
#pragma unroll
      for (int s = 0; s < ND; ++s) {
        uint4 e[2][3];
#pragma unroll
        for (int x = 0; x < 2; ++x) rows16<W>(te, 32 * jb + 16 * x, s, e[x]);
        dots_left16(e, y[s], p);
        dots_left16(e, z[s], r);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int j = 32 * jb + 16 * (e >> 2) + 4 * t4 + (e & 3);
        const float d = decay(my_sum - sums[j]) * rates[j];
        one[e] = j <= mine ? p[e >> 2][e & 3] * d * a.scale : 0.f;
        two[e] = j < mine ? -(r[e >> 2][e & 3] * d * my_rate) : 0.f;
        if (j == mine && t0 + mine < len) a.dbeta[row + t0 + mine] = r[e >> 2][e & 3];  // (z.E of one token)
      }
      uint4 op[3], tp[3];
      operand_of<3>(one, op);
      operand_of<3>(two, tp);
#pragma unroll
      for (int j = 0; j < 2 * ND; j += 2) {
        __builtin_amdgcn_sched_barrier(0);
        uint4 e[2][1];
        f32x4 w[2] = {dq[j], dq[j + 1]}, u[2] = {asked[j], asked[j + 1]};
#pragma unroll
        for (int x = 0; x < 2; ++x) columns16<L>(tk, 32 * jb, j + x, e[x]);
        dots_right16(op, e, w);
        dots_right16(tp, e, u);
        dq[j] = w[0], dq[j + 1] = w[1], asked[j] = u[0], asked[j + 1] = u[1];
      }
      settle_mfma();
    }
    // ---- the state before the block
    float early[4], rate[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) early[r] = decay(sums[own + 4 * t4 + r]), rate[r] = rates[own + 4 * t4 + r];
#pragma unroll
    for (int b = 0; b < ND; ++b)
      if (32 * b < a.dk) {
        const u16* const rows = next_rows(b);
        f32x4 of_y[2] = {zero4(), zero4()}, of_z[2] = {zero4(), zero4()};
#pragma unroll
        for (int s = 0; s < ND; ++s) {
          uint4 e[2][3];
#pragma unroll
          for (int x = 0; x < 2; ++x) rows16<Half>(rows, 16 * x, s, e[x]);
          dots_right16(y[s], e, of_y);
          dots_right16(z[s], e, of_z);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            dq[2 * b + x][r] = fmaf(of_y[x][r], early[r] * a.scale, dq[2 * b + x][r]);
            asked[2 * b + x][r] = fmaf(-of_z[x][r], early[r] * rate[r], asked[2 * b + x][r]);
          }
        settle_mfma();
      }
    float at[4] = {0.f, 0.f, 0.f, 0.f};  // q.dq + k.asked
#pragma unroll
    for (int j = 0; j < 2 * ND; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        at[r] = fmaf(tile_entry<L>(tq, own + 4 * t4 + r, 16 * j + l15), dq[j][r], at[r]);
        at[r] = fmaf(tile_entry<L>(tk, own + 4 * t4 + r, 16 * j + l15), asked[j][r], at[r]);
      }
    add_terms(at);
    __syncthreads();  // (the states have been read)
#pragma unroll
    for (int j = 0; j < 2 * ND; ++j) meet[j * 64 + lane] = asked[j];
    __syncthreads();
    by_rows<ND>(dq, buf, [&](int token, int c0, float (&x)[8]) { finish(0, token, c0, x); });
  } else {
    f32x4 kept[2 * ND];
#pragma unroll
    for (int j = 0; j < 2 * ND; ++j) kept[j] = zero4();
    uint4 e_own[ND][3];
#pragma unroll
    for (int s = 0; s < ND; ++s) rows16<W>(te, own, s, e_own[s]);
#pragma unroll 1
    for (int ib = own / 32; ib < 2; ++ib) {
      float one[8], two[8];
      f32x4 p[2] = {zero4(), zero4()}, r[2] = {zero4(), zero4()};
#pragma unroll
      for (int s = 0; s < ND; ++s) {
        uint4 y[2][1], z[2][3];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          rows16<L>(ty, 32 * ib + 16 * x, s, y[x]);
          rows16<W>(tz, 32 * ib + 16 * x, s, z[x]);
        }
        dots_left16(y, e_own[s], p);
        dots_left16(z, e_own[s], r);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = 32 * ib + 16 * (e >> 2) + 4 * t4 + (e & 3);
        const float d = decay(sums[i] - my_sum) * my_rate;
        one[e] = i >= mine ? p[e >> 2][e & 3] * d * a.scale : 0.f;
        two[e] = i > mine ? -(r[e >> 2][e & 3] * d * rates[i]) : 0.f;
      }
      uint4 op[3], tp[3];
      operand_of<3>(one, op);
      operand_of<3>(two, tp);
#pragma unroll
      for (int j = 0; j < 2 * ND; j += 2) {
        __builtin_amdgcn_sched_barrier(0);
        uint4 q[2][1], k[2][1];
        f32x4 u[2] = {kept[j], kept[j + 1]};
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          columns16<L>(tq, 32 * ib, j + x, q[x]);
          columns16<L>(tk, 32 * ib, j + x, k[x]);
        }
        dots_right16(op, q, u);
        dots_right16(tp, k, u);
        kept[j] = u[0], kept[j + 1] = u[1];
      }
      settle_mfma();
    }
    // ---- the gradient of the state behind the block
    const double end = sums[kBlock - 1];
    float late[4], late_terms = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) late[r] = decay(end - sums[own + 4 * t4 + r]) * rates[own + 4 * t4 + r];
#pragma unroll
    for (int b = 0; b < ND; ++b)
      if (32 * b < a.dk) {
        const u16* const rows = next_rows(b) + Half::kElems;
        f32x4 of_e[2] = {zero4(), zero4()};
#pragma unroll
        for (int s = 0; s < ND; ++s) {
          uint4 e[2][3];
#pragma unroll
          for (int x = 0; x < 2; ++x) rows16<Half>(rows, 16 * x, s, e[x]);
          dots_right16(e_own[s], e, of_e);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float e = of_e[x][r] * late[r];
            late_terms = fmaf(tile_entry<L>(tk, own + 4 * t4 + r, 32 * b + 16 * x + l15), e, late_terms);
            kept[2 * b + x][r] += e;
          }
        settle_mfma();
      }
    float at[4] = {0.f, 0.f, 0.f, 0.f};  // -k.kept
#pragma unroll
    for (int j = 0; j < 2 * ND; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) at[r] = fmaf(-tile_entry<L>(tk, own + 4 * t4 + r, 16 * j + l15), kept[j][r], at[r]);
    add_terms(at);
    inner = fmaf(inner, decay(end), late_terms);
    __syncthreads();
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2 * ND; ++j) kept[j] += meet[j * 64 + lane];
    by_rows<ND>(kept, buf, [&](int token, int c0, float (&x)[8]) { finish(1, token, c0, x); });
  }
  if (asks) inner *= decay(sums[kBlock - 1]);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) inner += __shfl_xor(inner, d);
  if (lane == 0) parts[wave] = inner;
  __syncthreads();
  if (wave == 0) {  // the gradient of g
    double sum = sum_from(terms[0][lane] + terms[1][lane]);
#pragma unroll
    for (int w = 0; w < 2 * kBackWaves; ++w) sum += parts[w];
    if (t0 + lane < len) a.dg[row + t0 + lane] = (float)sum;
  }
}

// dq and dk of query and key heads, sums over the value heads' in their order; zero behind a sequence.  x: entries at once.
template <typename T, int X>
__global__ void __launch_bounds__(256) delta_sums_kernel(DeltaArgs a, const float* sums) {
  const int64_t count = (int64_t)a.n * a.dk, heads = a.heads / a.G;
  const int shared = blockIdx.y % heads, which = blockIdx.y / heads;
  const int64_t end = (int64_t)tokens_of(a.lengths, shared / a.Hk, a.n) * a.dk;
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * X; i < count; i += (int64_t)gridDim.x * 256 * X) {
    const float* const from = sums + ((int64_t)which * a.heads + (int64_t)shared * a.G) * count + i;
    T* const to = (T*)(which ? a.dk_out : a.dq) + shared * count + i;
    float x[X] = {};
    if (i < end)
      for (int v = 0; v < a.G; ++v) {
        if constexpr (X == 4) {
          const float4 f = *(const float4*)(from + v * count);
          x[0] += f.x, x[1] += f.y, x[2] += f.z, x[3] += f.w;
        } else {
          x[0] += from[v * count];
        }
      }
    if constexpr (X == 4 && sizeof(T) == 2) *(uint2*)to = uint2{pack2(x[0], x[1]), pack2(x[2], x[3])};
    else if constexpr (X == 4) *(float4*)to = float4{x[0], x[1], x[2], x[3]};
    else to[0] = rounded<T>(x[0]);
  }
}

// Where a call's scratch goes.
struct Places {
  size_t data, back, states, behind, errors, zs, sums, bytes;
};
Places places_of(bool bf16, int heads, int G, int n, int dk, int dv) {
  const size_t blocks = (size_t)heads * ((n + kBlock - 1) / kBlock);
  auto whole = [](size_t x) { return (x + 255) / 256 * 256; };
  Places p;
  p.data = 0;
  p.back = whole(delta_forward_bytes(bf16, heads, n));
  p.states = p.back + whole(blocks * sizeof(DeltaBackward));
  p.behind = p.states + whole(blocks * dk * dv * sizeof(float));
  p.errors = p.behind + whole(blocks * dk * dv * sizeof(float));
  p.zs = p.errors + whole((size_t)heads * n * dv * sizeof(float));
  p.sums = p.zs + whole((size_t)heads * n * dv * sizeof(float));
  p.bytes = p.sums + (G > 1 ? 2 * (size_t)heads * n * dk * sizeof(float) : 0);
  return p;
}

template <typename F>
hipError_t raise_lds(F kern, int bytes) {
  return bytes > 60 * 1024 ? hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) : hipSuccess;
}

template <typename T, int ND>
hipError_t launch_scans(const DeltaArgs& a, const void* data, const void* back, float* states, float* behind, float* errors, float* zs,
                        hipStream_t s) {
  constexpr int bytes = std::max(BackLds<T, ND>::kBytes, DeltaLds<T, ND>::kBytes);
  auto kern = delta_scans_kernel<T, ND>;
  hipError_t e = raise_lds(kern, bytes);
  if (e != hipSuccess) return e;
  const int slices = (a.dv + 16 * kBackWaves - 1) / (16 * kBackWaves);
  hipLaunchKernelGGL(kern, dim3(2 * delta_grid(a.heads, slices)), dim3(kBackScanThreads), bytes, s, a, data, back, states, behind, errors, zs,
                     slices);
  return hipGetLastError();
}

template <typename T, int ND, bool MANY>
hipError_t launch_blocks_of(const DeltaArgs& a, const float* states, const float* behind, const float* errors, const float* zs,
                            float* sums, hipStream_t s) {
  const dim3 grid((a.n + kBlock - 1) / kBlock, a.heads);
  auto start = [&](auto kern, int threads, int bytes) {
    hipError_t e = raise_lds(kern, bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, grid, dim3(threads), bytes, s, a, states, behind, errors, zs, sums);
    return hipGetLastError();
  };
  if constexpr (sizeof(T) == 2) {
    static_assert(SplitLds<ND>::kBytes <= 158 * 1024, "LDS of one workgroup");
    return start(delta_split_kernel<ND, MANY>, kSplitThreads, SplitLds<ND>::kBytes);
  } else {
    static_assert(BlockLds<ND>::kBytes <= 158 * 1024, "LDS of one workgroup");
    return start(delta_blocks_kernel<ND, MANY>, kBackThreads, BlockLds<ND>::kBytes);
  }
}
template <typename T, int ND>
hipError_t launch_blocks(const DeltaArgs& a, const float* states, const float* behind, const float* errors, const float* zs,
                         float* sums, hipStream_t s) {
  if (a.G == 1) return launch_blocks_of<T, ND, false>(a, states, behind, errors, zs, sums, s);
  hipError_t e = launch_blocks_of<T, ND, true>(a, states, behind, errors, zs, sums, s);
  if (e != hipSuccess) return e;
  const bool fours = a.dk % 4 == 0 && (((uintptr_t)a.dq | (uintptr_t)a.dk_out) & (4 * sizeof(T) - 1)) == 0;
  const int64_t vectors = (int64_t)a.n * a.dk / (fours ? 4 : 1);
  const int rows = 2 * (a.heads / a.G);
  const dim3 grid((unsigned)std::min<int64_t>((vectors + 255) / 256, std::max(1, (1 << 22) / rows)), rows);
  if (fours) hipLaunchKernelGGL((delta_sums_kernel<T, 4>), grid, dim3(256), 0, s, a, sums);
  else hipLaunchKernelGGL((delta_sums_kernel<T, 1>), grid, dim3(256), 0, s, a, sums);
  return hipGetLastError();
}

template <typename T>
hipError_t launch(const DeltaArgs& a, char* scratch, hipStream_t s) {
  const Places p = places_of(sizeof(T) == 2, a.heads, a.G, a.n, a.dk, a.dv);
  float *states = (float*)(scratch + p.states), *behind = (float*)(scratch + p.behind);
  float *errors = (float*)(scratch + p.errors), *zs = (float*)(scratch + p.zs), *sums = (float*)(scratch + p.sums);
  const void *data = scratch + p.data, *back = scratch + p.back;
  hipError_t e = launch_delta_pairs(a, sizeof(T) == 2, scratch + p.data, scratch + p.back, s);
  if (e != hipSuccess) return e;
  switch ((a.dk + 31) / 32) {
    case 1: e = launch_scans<T, 1>(a, data, back, states, behind, errors, zs, s); break;
    case 2: e = launch_scans<T, 2>(a, data, back, states, behind, errors, zs, s); break;
    case 3: e = launch_scans<T, 3>(a, data, back, states, behind, errors, zs, s); break;
    default: e = launch_scans<T, 4>(a, data, back, states, behind, errors, zs, s); break;
  }
  if (e != hipSuccess) return e;
  switch ((std::max(a.dk, a.dv) + 31) / 32) {
    case 1: return launch_blocks<T, 1>(a, states, behind, errors, zs, sums, s);
    case 2: return launch_blocks<T, 2>(a, states, behind, errors, zs, sums, s);
    case 3: return launch_blocks<T, 3>(a, states, behind, errors, zs, sums, s);
    default: return launch_blocks<T, 4>(a, states, behind, errors, zs, sums, s);
  }
}

// No tokens: the states' gradients as they are.
__global__ void __launch_bounds__(256) delta_no_tokens_kernel(const float* dS, float* dS_in, int64_t count) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) dS_in[i] = dS ? dS[i] : 0.f;
}

}  // namespace

size_t delta_backward_scratch(bool bf16, int heads, int G, int n, int dk, int dv) {
  return n == 0 ? 0 : places_of(bf16, heads, G, n, dk, dv).bytes;
}

hipError_t launch_delta_backward(const DeltaArgs& a, bool bf16, void* scratch, hipStream_t s) {
  if (a.n == 0) {
    const int64_t count = (int64_t)a.heads * a.dk * a.dv;
    hipLaunchKernelGGL(delta_no_tokens_kernel, dim3((unsigned)std::min<int64_t>((count + 255) / 256, 65536)), dim3(256), 0, s, a.dS,
                       a.dS_in, count);
    return hipGetLastError();
  }
  return bf16 ? launch<u16>(a, (char*)scratch, s) : launch<float>(a, (char*)scratch, s);
}

}  // namespace sata
