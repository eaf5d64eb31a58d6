// Cross attention (hla_cross_attn_fwd, hla_cross_attn_bwd): queries against the states
// of another sequence, bf16 and fp32. For batch element b and key head t the keys
// j < length[b] are seen by the rows of the heads that share t:
//   S_rj = scale <q_r, k_j>,  P = softmax_j(S),  out_r = sum_j P_rj v_j,
//   lse_r = ln sum_j exp(S_rj),
// and backward, with delta_r = <dout_r, out_r>,
//   dS_rj = P_rj (<dout_r, v_j> - delta_r),
//   dq_r = scale sum_j dS_rj k_j,  dk_j = scale sum_r dS_rj q_r,  dv_j = sum_r P_rj dout_r.
//
// Rows. The heads that share a key head and their N queries form one list of G * N rows
// (row r is query r % N of head r / N), cut into tiles of 32 rows per wave: keys and
// values are read once for the whole group, a token's few heads fill one tile, and the
// sums over shared heads in dk and dv are sums over rows like any other.
//
// Forward: one workgroup per row tile; a wave keeps its 32 queries in registers and
// walks tiles of 64 keys that come into an LDS ring by the 16-byte LDS DMA, with the
// running maximum and sum of the softmax. Few rows against many keys: the keys are
// split over workgroups, whose partial sums (fp32, with their maxima) are joined by a
// second launch.
// Backward, two kernels as in the block-sparse backward, no atomics: dq per row tile
// (it also stores each row's statistics), then dk and dv per tile of 64 keys, the rows
// split over workgroups where there are few key tiles (fp32 partial sums, added in
// order by a third launch).
//
// Masked places: keys from length on are never loaded (the last tile's copies stop at
// the last seen key, of which the others are copies) and get weight 0, so nothing that
// stands there, NaN included, reaches a result.
#include <algorithm>

#include "cross_tiles.h"

namespace hla {
namespace {

constexpr int BN = 64;                // keys per tile
constexpr float kSlack = 8.f;         // log2 units the softmax reference may lag the max
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// ln of a row's sum (l, about the reference m in log2 units), and 1 / l. No key: l = 0
// gives -inf and 0. (NaN stays NaN.)
__device__ __forceinline__ float lse_of(float m, float l) {
  return l == 0.f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * kLn2;
}
__device__ __forceinline__ float inv_of(float l) { return l == 0.f ? 0.f : 1.f / l; }

struct Row {
  int head, n;
};
__device__ __forceinline__ Row row_of(const CrossArgs &a, int r, int kvh) {
  const int g = (int)fdiv((uint32_t)r, a.ndiv);
  return {kvh * a.G + g, r - g * a.N};
}
template <typename T>
__device__ __forceinline__ T *row_ptr(const void *p, const CrossStride &s, int b, const Row &r) {
  return const_cast<T *>(static_cast<const T *>(p)) + b * s.batch + r.head * s.head + r.n * s.row;
}

// Keys seen by batch element b.
__device__ __forceinline__ int keys_of(const CrossArgs &a, int b) {
  return a.lengths ? clampi(sload(a.lengths + b), 0, a.M) : a.M;
}

// Copies of 64 rows from row 0 of K and V on into a stage (K tile, then V tile); rows
// past `last` read row last. kr, vr: bytes between rows.
template <typename T, int D, int NW>
struct KvCopy {
  using Tl = Tile<T, D>;
  static constexpr int CPW = BN * Tl::CPR / (64 * NW), LPT = 2 * CPW;
  static_assert(BN * Tl::CPR % (64 * NW) == 0, "copies must split evenly");
  static __device__ __forceinline__ void issue(const char *K, const char *V, uint32_t kr, uint32_t vr, int last,
                                               char *stage, int wave, int lane) {
#pragma unroll
    for (int j = 0; j < CPW; ++j) {
      const int p = (j * NW + wave) * 64 + lane, r = p / Tl::CPR, c = (p % Tl::CPR) ^ Tl::swz(r);
      lds_dma16_at(K, (uint32_t)min(r, last) * kr + c * 16, lds_addr(stage + (j * NW + wave) * 1024));
    }
#pragma unroll
    for (int j = 0; j < CPW; ++j) {
      const int p = (j * NW + wave) * 64 + lane, r = p / Tl::CPR, c = (p % Tl::CPR) ^ Tl::swz(r);
      lds_dma16_at(V, (uint32_t)min(r, last) * vr + c * 16, lds_addr(stage + BN * Tl::ROW + (j * NW + wave) * 1024));
    }
  }
};

// Scores of the keys from `left` on (slot v of lane half `half`: key
// 16 (v/8) + 8 half + v%8 of the block) become -inf.
__device__ __forceinline__ void mask_tail(f32x16 &s, int left, int half) {
#pragma unroll
  for (int v = 0; v < 16; ++v)
    s[v] = 16 * (v >> 3) + 8 * half + (v & 7) < left ? s[v] : -__builtin_inff();
}

template <typename T, int D>
constexpr int fwd_ring() { return sizeof(T) == 4 ? 2 : 3; }

template <typename T, int D, int NW>
__global__ void __launch_bounds__(64 * NW, NW == 1 ? 1 : 2) cross_fwd(CrossArgs a) {
  using Tl = Tile<T, D>;
  constexpr int NDB = Tl::NDB, RING = fwd_ring<T, D>();
  constexpr int STAGE = 2 * BN * Tl::ROW;
  constexpr int AREA = 32 * (Tl::ROW + 16);
  static_assert(NW * AREA <= RING * STAGE, "the rows' staging must fit the ring");
  using Copy = KvCopy<T, D, NW>;
  static_assert(Copy::LPT * (RING - 2) < 64, "vmcnt range");
  __shared__ __attribute__((aligned(16))) char lds[RING * STAGE];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int logical = xcd_remap(blockIdx.x, gridDim.x);
  const int rt = logical % a.n_rtiles, t = logical / a.n_rtiles;
  const int sp = t % a.splits, bk = t / a.splits, b = bk / a.kv, kvh = bk - b * a.kv;

  // This split's keys [k0, k1): whole tiles but for the last.
  const int len = keys_of(a, b);
  const int per = (((len + a.splits - 1) / a.splits) + BN - 1) / BN * BN;
  const int k0 = min(sp * per, len), k1 = min(k0 + per, len);
  const int nt = (k1 - k0 + BN - 1) / BN;
  const char *K = reinterpret_cast<const char *>(static_cast<const T *>(a.k) + b * a.ks.batch + kvh * a.ks.head);
  const char *V = reinterpret_cast<const char *>(static_cast<const T *>(a.v) + b * a.vs.batch + kvh * a.vs.head);
  const uint32_t kr = (uint32_t)a.ks.row * sizeof(T), vr = (uint32_t)a.vs.row * sizeof(T);
  auto issue = [&](int i) {
    const int at = k0 + i * BN;
    Copy::issue(K + (int64_t)at * kr, V + (int64_t)at * vr, kr, vr, k1 - 1 - at, lds + (i % RING) * STAGE, wave, lane);
  };
#pragma unroll
  for (int i = 0; i < RING - 1; ++i)
    if (i < nt) issue(i);

  // (rows past the last read it and store nothing)
  const int r0 = (rt * NW + wave) * 32, r = r0 + col;
  const Row rw = row_of(a, min(r, a.R - 1), kvh);
  typename Tl::Frag q;
  Tl::load(q, row_ptr<T>(a.q, a.qs, b, rw), half);
  Tl tl;
  tl.init(lane);
  f32x16 o[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) o[db] = f32x16{};
  float m = -__builtin_inff(), l = 0.f;   // reference (log2 units), this lane's half of the sum
  wait_vmem_all();

  for (int i = 0; i < nt; ++i) {
    wait_tiles_then_barrier<Copy::LPT, RING - 2>(min(RING - 2, nt - 1 - i));
    if (i + RING - 1 < nt) issue(i + RING - 1);
    const char *st = lds + (i % RING) * STAGE;
    const int left = k1 - (k0 + i * BN);   // keys of this tile, and beyond
    // Both blocks of 32 keys together; a last tile of one block leaves the other out.
    f32x16 s[2];
    const bool two = left > 32;
    tl.rows_times(st, q, s[0]);
    if (two) tl.rows_times(st + 32 * Tl::ROW, q, s[1]);
    if (left < BN) {
      if (two) mask_tail(s[1], left - 32, half);
      else mask_tail(s[0], left, half);
    }
    float mx = s[0][0];
#pragma unroll
    for (int v = 1; v < 16; ++v) mx = fmaxf(mx, s[0][v]);
    if (two) {
#pragma unroll
      for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[1][v]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 32)) * a.scale_log2;
    // The reference moves only when the tile's max passes it by the slack (weights
    // stay <= 2^8; O and l share it).
    const bool need = mx > m + kSlack;
    if (__ballot(need)) {
      const float m_new = need ? mx : m, alpha = need ? __builtin_amdgcn_exp2f(m - m_new) : 1.f;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < NDB; ++db) o[db] *= alpha;
      m = m_new;
    }
    const float ref = m == -__builtin_inff() ? 0.f : m;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      if (kb == 1 && !two) break;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        s[kb][v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][v], a.scale_log2, -ref));
        l += s[kb][v];
      }
      tl.cols_times(st + BN * Tl::ROW + kb * 32 * Tl::ROW, s[kb], o);
    }
  }
  l += __shfl_xor(l, 32);

  if (a.splits > 1) {
    const int64_t at = ((int64_t)bk * a.splits + sp) * a.R + r;
    if (r < a.R) {
      float *p = a.part + at * D;
      Tl::columns(o, half, [&](int c, f32x4 v) { *reinterpret_cast<f32x4 *>(p + c) = v; });
      if (half == 0) a.part_ml[at] = make_float2(m, l);
    }
    return;
  }
  wait_then_barrier<0>();   // every wave is done with the ring
  const int64_t first = ((int64_t)b * a.kv + kvh) * a.R;   // = (b * heads + kvh * G) * N
  if (a.lse && half == 0 && r < a.R) a.lse[first + r] = lse_of(m, l);
  const float inv = inv_of(l);
  // each lane's factor goes into its own row before the rows are staged
#pragma unroll
  for (int db = 0; db < NDB; ++db) o[db] *= inv;
  store_rows<T, D>(lds + wave * AREA, o, 1.f, lane, [&](int i) {
    return r0 + i < a.R ? row_ptr<T>(a.out, a.os, b, row_of(a, r0 + i, kvh)) : nullptr;
  });
}

// Joins the partial sums of the key splits: one thread per row and four columns.
template <typename T, int D>
__global__ void __launch_bounds__(256) cross_join(CrossArgs a) {
  constexpr int TPR = D / 4;
  const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = idx / TPR;
  if (row >= (int64_t)a.B * a.kv * a.R) return;
  const int c = (int)(idx % TPR) * 4;
  const int bk = (int)(row / a.R), r = (int)(row - (int64_t)bk * a.R), b = bk / a.kv, kvh = bk - b * a.kv;
  const float2 *ml = a.part_ml + (int64_t)bk * a.splits * a.R + r;
  const float *p = a.part + ((int64_t)bk * a.splits * a.R + r) * D + c;
  float m = -__builtin_inff();
  for (int s = 0; s < a.splits; ++s) m = fmaxf(m, ml[(int64_t)s * a.R].x);
  const float ref = m == -__builtin_inff() ? 0.f : m;
  float l = 0.f;
  f32x4 o = {};
  for (int s = 0; s < a.splits; ++s) {
    const float2 e = ml[(int64_t)s * a.R];
    const f32x4 x = *reinterpret_cast<const f32x4 *>(p + (int64_t)s * a.R * D);
    const float w = __builtin_amdgcn_exp2f(e.x - ref);
    l += w * e.y;
    o += w * x;
  }
  if (a.lse && c == 0) a.lse[(int64_t)bk * a.R + r] = lse_of(m, l);
  put4<T>(row_ptr<T>(a.out, a.os, b, row_of(a, r, kvh)) + c, o * inv_of(l));
}

// dq, and the rows' statistics for the next kernel: lse log2 e (+inf for a row without
// a key and for the padding of the last tile, which makes every weight exp2(s - inf) =
// 0) and -delta.
template <typename T, int D, int NW>
__global__ void __launch_bounds__(64 * NW, 2) cross_dq(CrossArgs a) {
  using Tl = Tile<T, D>;
  constexpr int NDB = Tl::NDB, RING = fwd_ring<T, D>();
  constexpr int STAGE = 2 * BN * Tl::ROW;
  constexpr int AREA = 32 * (Tl::ROW + 16);
  using Copy = KvCopy<T, D, NW>;
  __shared__ __attribute__((aligned(16))) char lds[RING * STAGE];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int logical = xcd_remap(blockIdx.x, gridDim.x);
  const int rt = logical % a.n_rtiles, bk = logical / a.n_rtiles, b = bk / a.kv, kvh = bk - b * a.kv;
  const int len = keys_of(a, b), nt = (len + BN - 1) / BN;
  const char *K = reinterpret_cast<const char *>(static_cast<const T *>(a.k) + b * a.ks.batch + kvh * a.ks.head);
  const char *V = reinterpret_cast<const char *>(static_cast<const T *>(a.v) + b * a.vs.batch + kvh * a.vs.head);
  const uint32_t kr = (uint32_t)a.ks.row * sizeof(T), vr = (uint32_t)a.vs.row * sizeof(T);
  auto issue = [&](int i) {
    const int at = i * BN;
    Copy::issue(K + (int64_t)at * kr, V + (int64_t)at * vr, kr, vr, len - 1 - at, lds + (i % RING) * STAGE, wave, lane);
  };
#pragma unroll
  for (int i = 0; i < RING - 1; ++i)
    if (i < nt) issue(i);

  const int r0 = (rt * NW + wave) * 32, r = r0 + col;
  const Row rw = row_of(a, min(r, a.R - 1), kvh);
  typename Tl::Frag q, g;
  Tl::load(q, row_ptr<T>(a.q, a.qs, b, rw), half);
  Tl::load(g, row_ptr<T>(a.dout, a.gs, b, rw), half);
  float lse2, ndelta;
  {
    typename Tl::Frag out;
    Tl::load(out, row_ptr<T>(a.out, a.os, b, rw), half);
    const float lraw = a.lse[(int64_t)bk * a.R + min(r, a.R - 1)];
    wait_vmem_all();
    const float d = Tl::dot(out, g);
    ndelta = -(d + __shfl_xor(d, 32));
    lse2 = r < a.R && lraw != -__builtin_inff() ? lraw * kLog2e : __builtin_inff();
  }
  if (half == 0) {
    const int64_t at = (int64_t)bk * a.Rp + r;
    a.stats[at] = lse2;
    a.stats[(int64_t)a.B * a.kv * a.Rp + at] = ndelta;
  }
  Tl tl;
  tl.init(lane);
  f32x16 acc[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) acc[db] = f32x16{};

  for (int i = 0; i < nt; ++i) {
    wait_tiles_then_barrier<Copy::LPT, RING - 2>(min(RING - 2, nt - 1 - i));
    if (i + RING - 1 < nt) issue(i + RING - 1);
    const char *st = lds + (i % RING) * STAGE;
    const int left = len - i * BN;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      if (32 * kb >= left) break;
      const char *blk = st + kb * 32 * Tl::ROW;
      f32x16 s, dp;
      tl.rows_times(blk, q, s);
      tl.rows_times(blk + BN * Tl::ROW, g, dp);
      if (left < 32 * kb + 32) mask_tail(s, left - 32 * kb, half);
#pragma unroll
      for (int v = 0; v < 16; ++v)
        s[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[v], a.scale_log2, -lse2)) * (dp[v] + ndelta);
      tl.cols_times(blk, s, acc);
    }
  }
  wait_then_barrier<0>();
  store_rows<T, D>(lds + wave * AREA, acc, a.scale, lane, [&](int i) {
    return r0 + i < a.R ? row_ptr<T>(a.dq, a.dqs, b, row_of(a, r0 + i, kvh)) : nullptr;
  });
}

// dk and dv of 64 keys. Wave w takes the 32 keys of block w % 2 against half w / 2 of
// the rows of every step (RB blocks of 32); the halves are added through LDS.
template <typename T, int D, int RB>
__global__ void __launch_bounds__(256, 2) cross_dkdv(CrossArgs a) {
  using Tl = Tile<T, D>;
  constexpr int NDB = Tl::NDB, BR = 64 * RB;   // rows per step
  constexpr int TILE = BR * Tl::ROW;
  constexpr int STAT = 2 * TILE, STAGE = STAT + BR * 8;
  constexpr int CPW = BR * Tl::CPR / 256;
  constexpr int AREA = 32 * (Tl::ROW + 16);
  constexpr int XCH = 2 * 2 * NDB * 16 * 64 * 4;
  constexpr int LDSB = 2 * STAGE > XCH ? 2 * STAGE : XCH;
  static_assert(4 * AREA <= LDSB, "the rows' staging must fit the ring");
  __shared__ __attribute__((aligned(16))) char lds[LDSB];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5, kb = wave & 1, rh = wave >> 1;
  const int logical = xcd_remap(blockIdx.x, gridDim.x);
  const int kt = logical % a.n_ktiles, t = logical / a.n_ktiles;
  const int sp = t % a.splits, bk = t / a.splits, b = bk / a.kv, kvh = bk - b * a.kv;
  const int len = keys_of(a, b);
  const int kpos = kt * BN + 32 * kb + col;
  // (no key of the tile is seen: zeros, which the joining launch knows by itself)
  if (kt * BN >= len && a.splits > 1) return;

  // This split's rows [r0, r1): whole steps but for the last.
  const int steps = (a.R + BR - 1) / BR, per = (steps + a.splits - 1) / a.splits;
  const int i0 = min(sp * per, steps), i1 = kt * BN < len ? min(i0 + per, steps) : i0;
  const float *S = a.stats + (int64_t)bk * a.Rp;
  const int64_t dofs = (int64_t)a.B * a.kv * a.Rp;   // from lse to -delta
  auto issue = [&](int i) {
    char *stage = lds + (i & 1) * STAGE;
#pragma unroll
    for (int j = 0; j < CPW; ++j) {
      const int p = (j * 4 + wave) * 64 + lane, rr = p / Tl::CPR, c = (p % Tl::CPR) ^ Tl::swz(rr);
      // (rows past the last read it; their statistics make their weights 0)
      const Row rw = row_of(a, min(i * BR + rr, a.R - 1), kvh);
      lds_dma16(reinterpret_cast<const char *>(row_ptr<T>(a.q, a.qs, b, rw)) + c * 16, lds_addr(stage + (j * 4 + wave) * 1024));
      lds_dma16(reinterpret_cast<const char *>(row_ptr<T>(a.dout, a.gs, b, rw)) + c * 16,
                lds_addr(stage + TILE + (j * 4 + wave) * 1024));
    }
    if (wave < 2 * RB) {   // 64 rows' lse, or -delta, per wave
      const int which = wave / RB, part = wave % RB;
      lds_dma4(S + which * dofs + i * BR + part * 64 + lane, lds_addr(stage + STAT + which * BR * 4 + part * 256));
    }
  };
  if (i0 < i1) issue(i0);

  const int64_t krow = min(kpos, max(len - 1, 0));   // (unseen keys: not stored)
  typename Tl::Frag k, v;
  Tl::load(k, static_cast<const T *>(a.k) + b * a.ks.batch + kvh * a.ks.head + krow * a.ks.row, half);
  Tl::load(v, static_cast<const T *>(a.v) + b * a.vs.batch + kvh * a.vs.head + krow * a.vs.row, half);
  Tl tl;
  tl.init(lane);
  f32x16 dk[NDB], dv[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) dk[db] = dv[db] = f32x16{};
  wait_vmem_all();

  for (int i = i0; i < i1; ++i) {
    wait_then_barrier<0>();
    if (i + 1 < i1) issue(i + 1);
    const char *st = lds + (i & 1) * STAGE;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int first = (rh * RB + rb) * 32;
      const char *blk = st + first * Tl::ROW;
      const float *stat = reinterpret_cast<const float *>(st + STAT) + first + 8 * half;
      f32x16 s, dp;
      tl.rows_times(blk, k, s);
      tl.rows_times(blk + TILE, v, dp);
#pragma unroll
      for (int x = 0; x < 4; ++x) {   // slots 4x .. 4x + 3: rows 16 (x/2) + 4 (x%2) ..
        const f32x4 l4 = *reinterpret_cast<const f32x4 *>(stat + 16 * (x >> 1) + 4 * (x & 1));
        const f32x4 d4 = *reinterpret_cast<const f32x4 *>(stat + BR + 16 * (x >> 1) + 4 * (x & 1));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * x + e], a.scale_log2, -l4[e]));
          s[4 * x + e] = p;
          dp[4 * x + e] = p * (dp[4 * x + e] + d4[e]);
        }
      }
      tl.cols_times(blk + TILE, s, dv);
      tl.cols_times(blk, dp, dk);
    }
  }

  // Half 1 hands its dk to half 0, half 0 its dv to half 1; then half 0 has dk, half 1 dv.
  wait_then_barrier<0>();
  float *xch = reinterpret_cast<float *>(lds);
  auto at = [&](int which, int db, int e) { return (((kb * 2 + which) * NDB + db) * 16 + e) * 64 + lane; };
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) xch[at(rh, db, e)] = rh ? dk[db][e] : dv[db][e];
  wait_then_barrier<0>();
  f32x16 sum[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) sum[db][e] = (rh ? dv[db][e] : dk[db][e]) + xch[at(1 - rh, db, e)];
  wait_then_barrier<0>();
  if (a.splits > 1) {
    if (kpos < len) {
      float *p = a.part + ((((int64_t)sp * a.B * a.kv + bk) * a.M + kpos) * 2 + rh) * D;
      Tl::columns(sum, half, [&](int c, f32x4 x) { *reinterpret_cast<f32x4 *>(p + c) = x; });
    }
    return;
  }
  if (kpos >= len) {
#pragma unroll
    for (int db = 0; db < NDB; ++db) sum[db] = f32x16{};
  }
  const CrossStride &os = rh ? a.dvs : a.dks;
  T *dst = static_cast<T *>(rh ? a.dv : a.dk) + b * os.batch + kvh * os.head;
  const int j0 = kt * BN + 32 * kb;
  store_rows<T, D>(lds + wave * AREA, sum, rh ? 1.f : a.scale, lane,
                   [&](int i) { return j0 + i < a.M ? dst + (j0 + i) * os.row : nullptr; });
}

// Adds the partial sums of the row splits: one thread per key, gradient and four columns.
template <typename T, int D>
__global__ void __launch_bounds__(256) cross_sum(CrossArgs a) {
  constexpr int TPR = D / 4;
  const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int c = (int)(idx % TPR) * 4, which = (int)(idx / TPR % 2);
  const int64_t key = idx / (2 * TPR), keys = (int64_t)a.B * a.kv * a.M;
  if (key >= keys) return;
  const int bk = (int)(key / a.M), j = (int)(key - (int64_t)bk * a.M), b = bk / a.kv, kvh = bk - b * a.kv;
  f32x4 sum = {};
  if (j < keys_of(a, b)) {
    const float *p = a.part + (key * 2 + which) * D + c;
    for (int s = 0; s < a.splits; ++s) sum += *reinterpret_cast<const f32x4 *>(p + s * keys * 2 * D);
  }
  const CrossStride &os = which ? a.dvs : a.dks;
  T *dst = static_cast<T *>(which ? a.dv : a.dk) + b * os.batch + kvh * os.head + j * os.row;
  put4<T>(dst + c, sum * (which ? 1.f : a.scale));
}

// Row tiles of one wave where a list's rows fit one: its workgroups are then single
// waves, each with a ring of its own.
int fwd_waves(const CrossArgs &a) { return a.R <= 32 ? 1 : 4; }

template <typename T, int D>
hipError_t fwd(CrossArgs &a, hipStream_t s) {
  const int nw = fwd_waves(a);
  a.n_rtiles = (a.R + 32 * nw - 1) / (32 * nw);
  const dim3 grid((uint32_t)((int64_t)a.B * a.kv * a.n_rtiles * a.splits));
  if (nw == 1) hipLaunchKernelGGL((cross_fwd<T, D, 1>), grid, dim3(64), 0, s, a);
  else hipLaunchKernelGGL((cross_fwd<T, D, 4>), grid, dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t n = (int64_t)a.B * a.kv * a.R * (D / 4);
  hipLaunchKernelGGL((cross_join<T, D>), dim3((uint32_t)((n + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t bwd(CrossArgs &a, hipStream_t s) {
  constexpr int RB = sizeof(T) == 4 ? 1 : 2;
  a.n_rtiles = (a.R + 127) / 128;
  hipLaunchKernelGGL((cross_dq<T, D, 4>), dim3((uint32_t)((int64_t)a.B * a.kv * a.n_rtiles)), dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((cross_dkdv<T, D, RB>), dim3((uint32_t)((int64_t)a.B * a.kv * a.n_ktiles * a.splits)), dim3(256), 0, s, a);
  e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t n = (int64_t)a.B * a.kv * a.M * 2 * (D / 4);
  hipLaunchKernelGGL((cross_sum<T, D>), dim3((uint32_t)((n + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

int up_to(int64_t want, int64_t most) { return (int)std::max<int64_t>(1, std::min(want, most)); }

}  // namespace

// Key splits of the forward: enough workgroups to fill the chip with 8 waves per CU,
// but at least two tiles of keys each.
int cross_fwd_splits(const CrossArgs &a) {
  const int nw = fwd_waves(a);
  const int64_t wgs = (int64_t)a.B * a.kv * ((a.R + 32 * nw - 1) / (32 * nw));
  return up_to((int64_t)device_cu_count() * 8 / nw / wgs, (a.M + 2 * BN - 1) / (2 * BN));
}

// Row splits of dk and dv: two workgroups per CU, at least four steps of 64 rows each.
int cross_bwd_splits(const CrossArgs &a) {
  const int64_t wgs = (int64_t)a.B * a.kv * ((a.M + BN - 1) / BN);
  return up_to((int64_t)device_cu_count() * 2 / wgs, (a.R + 255) / 256);
}

hipError_t launch_cross_fwd(CrossArgs a, int d, hla_dtype dtype, hipStream_t s) {
  if (dtype == HLA_BF16) return d == 32 ? fwd<__bf16, 32>(a, s) : fwd<__bf16, 64>(a, s);
  return d == 32 ? fwd<float, 32>(a, s) : fwd<float, 64>(a, s);
}
hipError_t launch_cross_bwd(CrossArgs a, int d, hla_dtype dtype, hipStream_t s) {
  if (dtype == HLA_BF16) return d == 32 ? bwd<__bf16, 32>(a, s) : bwd<__bf16, 64>(a, s);
  return d == 32 ? bwd<float, 32>(a, s) : bwd<float, 64>(a, s);
}

}  // namespace hla
