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
// Forward, by shape:
//  many rows    a workgroup per 128 rows; a wave keeps its 32 queries in registers, and the
//               four walk tiles of 64 keys that come into an LDS ring by the 16-byte LDS
//               DMA, with the running maximum and sum of the softmax;
//  few rows     a workgroup per 32 rows, its waves on tiles of their own, and the keys split
//               over workgroups too, whose partial sums (fp32, with their maxima) a second
//               launch joins;
//  few keys     keys and values stay in LDS, and the waves go through blocks of 32 rows.
// Backward, two kernels as in the block-sparse backward, no atomics: dq in the same three
// ways (it also stores each row's statistics), then dk and dv per tile of 64 or 128 keys,
// the rows split over workgroups where there are few key tiles (fp32 partial sums, added
// in order by a third launch).
//
// What bounds them, in heads of 64 with many rows and keys: a wave's exponentials and its
// matrix products follow one another, and too few waves stand beside it: 512 workgroups of
// four are two to a SIMD, 1.6 of them resident over the launch (1.2 where lengths are ragged).
// 8 heads on 2, 4096 rows and keys, batch 2, bf16, by the clock: forward 101 to 117 us (590
// to 680 TFLOP/s; vector issue 49%, matrix cores 26%), dq 115 to 130 (790 to 890; 48, 36%), dk
// and dv 139 to 153 (900 to 990; 46, 42%).
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
constexpr float kWindow = 4096.f;     // weights about a reference that no maximum was taken for, per key
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// ln of a row's sum (l, about the reference m in log2 units), and 1 / l. No key: l = 0
// gives -inf and 0. (NaN stays NaN.)
__device__ __forceinline__ float lse_of(float m, float l) {
  return l == 0.f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * kLn2;
}
__device__ __forceinline__ float inv_of(float l) { return l == 0.f ? 0.f : 1.f / l; }

// Row r of key head kvh: query n of a head.
struct Row {
  uint32_t head, n;
};
__device__ __forceinline__ Row row_of(const CrossArgs &a, int r, int kvh) {
  if (a.G == 1) return {(uint32_t)kvh, (uint32_t)r};
  const uint32_t g = fdiv((uint32_t)r, a.ndiv);
  return {kvh * a.G + g, r - g * a.N};
}
// Its address: 32-bit arithmetic in units of 16 bytes within the batch element.
template <typename T>
__device__ __forceinline__ T *row_ptr(const void *p, const CrossStride &s, int b, const Row &r) {
  char *base = static_cast<char *>(const_cast<void *>(p)) + b * s.batch;
  return reinterpret_cast<T *>(base + ((uint64_t)(r.head * s.head + r.n * s.row) << 4));
}
// The first row of key head kvh.
__device__ __forceinline__ const char *head_ptr(const void *p, const CrossStride &s, int b, int kvh) {
  return static_cast<const char *>(p) + b * s.batch + ((uint64_t)(kvh * s.head) << 4);
}

// Workgroup -> piece of work. The pieces are ordered by (batch, key head), whose keys they
// share, and workgroups go round-robin over the 8 XCDs: runs of `unit` consecutive
// pieces are dealt to the XCDs in turn, so that a run shares its keys in one L2 while
// every XCD gets its part of the long and of the short batch elements. (Lengths 4096 and
// about 2000, 16384 rows each: one contiguous range per XCD leaves half the chip
// with the long element.) total = pieces; past them the result is >= total.
__device__ __forceinline__ int deal(int bid, int unit) {
  const int xcd = bid & 7, slot = bid >> 3, u = slot / unit;
  return (u * 8 + xcd) * unit + slot - u * unit;
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

// The running softmax of a wave's 32 rows: reference m (log2 units), this lane's half of
// the sum l about it, O^T about it.
template <typename T, int D>
struct Softmax {
  using Tl = Tile<T, D>;
  f32x16 o[Tl::NDB];
  float m, l;
  bool primed;   // every row of the wave has a finite reference
  bool fresh;    // no key yet

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int db = 0; db < Tl::NDB; ++db) o[db] = f32x16{};
    m = -__builtin_inff();
    l = 0.f;
    primed = false;
    fresh = true;
  }
  // weights of NB blocks in place of their scores; returns the new sum. NV = 8: only
  // the first 16 keys are seen (a lane's first eight slots).
  template <int NB, int NV = 16>
  __device__ __forceinline__ float weights(f32x16 (&s)[NB], float scale, float ref) const {
    float sum[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) sum[b] = b ? 0.f : l;
#pragma unroll
    for (int v = 0; v < 16; ++v)
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        if (v >= NV) {
          s[b][v] = 0.f;
          continue;
        }
        s[b][v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][v], scale, -ref));
        sum[b] += s[b][v];
      }
    return NB == 2 ? sum[0] + sum[NB - 1] : sum[0];
  }
  // NB blocks of 32 keys at k and v; TAIL: keys from `left` on are not seen. Once all
  // references are finite the weights are taken against them as they stand, with no
  // maximum: as all are >= 0, their sum of at most kWindow a key (NaN and inf fail it too)
  // accepts them in one compare. The first keys try the reference 0 in the same way, with a
  // lower bound as well. Only where that fails are the scores formed again and the
  // reference moved, if a score passes it by more than the slack. So a row's weights sum to
  // at most 2^12 M, and O stays in range for |v| up to 2^116 / M. (A window of 2^8 costs
  // time where scores are a few times wider than of unit normal q and k: 4096 rows and keys
  // of 64, q of deviation 2, 104.5 us against 100.7; one of 2^16 gains nothing there. At
  // deviation 4 and 77 keys, most first tries fail: 21.6 us, and 18.0 with a window of 2^32.)
  template <int NB, bool TAIL>
  __device__ __forceinline__ void step(const Tl &tl, const char *k, const char *v, const typename Tl::Frag &q,
                                       float scale, int left, int half) {
    f32x16 s[NB];
    auto scores = [&]() {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        tl.rows_times(k + b * 32 * Tl::ROW, q, s[b]);
        if (TAIL) mask_tail(s[b], left - 32 * b, half);
      }
    };
    scores();
    float ln = 0.f;
    bool slow = !primed;
    if (primed || fresh) {
      ln = TAIL && left <= 16 ? weights<NB, 8>(s, scale, fresh ? 0.f : m) : weights(s, scale, fresh ? 0.f : m);
      // (16 NB: the keys of a lane)
      const bool bad = !(ln - l <= 16 * NB * kWindow) || (fresh && !(ln >= 1.f / kWindow));
      slow = false;
      if (!__ballot(bad)) {
        if (fresh) m = 0.f;
        primed = true;
      } else {
        slow = true;
        asm volatile("" ::: "memory");   // (read the keys again rather than keep them in registers)
        scores();
      }
    }
    if (slow) {
      float mx = s[0][0];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[b][e]);
      mx = fmaxf(mx, __shfl_xor(mx, 32)) * scale;
      const bool need = mx > m + kSlack;
      if (__ballot(need)) {
        const float m_new = need ? mx : m, alpha = need ? __builtin_amdgcn_exp2f(m - m_new) : 1.f;
        l *= alpha;
#pragma unroll
        for (int db = 0; db < Tl::NDB; ++db) o[db] *= alpha;
        m = m_new;
      }
      ln = weights(s, scale, m == -__builtin_inff() ? 0.f : m);
      primed = !__ballot(m == -__builtin_inff());
    }
    fresh = false;
    l = ln;
#pragma unroll
    for (int b = 0; b < NB; ++b) tl.cols_times(v + b * 32 * Tl::ROW, s[b], o);
  }
  // a tile of 64 keys, `left` of them (and of what follows) seen
  __device__ __forceinline__ void tile(const Tl &tl, const char *k, const char *v, const typename Tl::Frag &q,
                                       float scale, int left, int half) {
    if (left >= BN) {
      step<2, false>(tl, k, v, q, scale, left, half);
    } else {
#pragma unroll 1
      for (int b = 0; 32 * b < left; ++b)
        step<1, true>(tl, k + b * 32 * Tl::ROW, v + b * 32 * Tl::ROW, q, scale, left - 32 * b, half);
    }
  }
};

template <typename T, int D>
constexpr int fwd_ring() { return sizeof(T) == 4 ? 2 : 3; }

// Many rows: one workgroup per tile of 128 rows, its four waves on the same key tiles.
template <typename T, int D>
__global__ void __launch_bounds__(256, 2) cross_fwd(CrossArgs a) {
  using Tl = Tile<T, D>;
  constexpr int NDB = Tl::NDB, RING = fwd_ring<T, D>(), NW = 4;
  constexpr int STAGE = 2 * BN * Tl::ROW;
  constexpr int AREA = 32 * (Tl::ROW + 16);
  static_assert(NW * AREA <= RING * STAGE, "the rows' staging must fit the ring");
  using Copy = KvCopy<T, D, NW>;
  static_assert(Copy::LPT < 64, "vmcnt range");
  __shared__ __attribute__((aligned(16))) char lds[RING * STAGE];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int logical = deal(blockIdx.x, a.unit);
  if (logical >= a.total) return;
  const int rt = logical % a.n_rtiles, bk = logical / a.n_rtiles, b = bk / a.kv, kvh = bk - b * a.kv;
  const int len = keys_of(a, b), nt = (len + BN - 1) / BN;
  const char *K = head_ptr(a.k, a.ks, b, kvh), *V = head_ptr(a.v, a.vs, b, kvh);
  const uint32_t kr = a.ks.row * 16, vr = a.vs.row * 16;
  auto issue = [&](int i) {
    const int at = i * BN;
    Copy::issue(K + (int64_t)at * kr, V + (int64_t)at * vr, kr, vr, len - 1 - at, lds + (i % RING) * STAGE, wave, lane);
  };
#pragma unroll
  for (int i = 0; i < RING - 1; ++i)
    if (i < nt) issue(i);

  // (rows past the last read it and store nothing)
  const int r0 = (rt * NW + wave) * 32, r = r0 + col;
  typename Tl::Frag q;
  Tl::load(q, row_ptr<T>(a.q, a.qs, b, row_of(a, min(r, a.R - 1), kvh)), half);
  Tl tl;
  tl.init(lane);
  Softmax<T, D> sm;
  sm.init();
  wait_vmem_all();

  for (int i = 0; i < nt; ++i) {
    wait_tiles_then_barrier<Copy::LPT, RING - 2>(min(RING - 2, nt - 1 - i));
    if (i + RING - 1 < nt) issue(i + RING - 1);
    const char *st = lds + (i % RING) * STAGE;
    sm.tile(tl, st, st + BN * Tl::ROW, q, a.scale_log2, len - i * BN, half);
  }
  const float l = sm.l + __shfl_xor(sm.l, 32);
  wait_then_barrier<0>();   // every wave is done with the ring
  if (a.lse && half == 0 && r < a.R) a.lse[(int64_t)bk * a.R + r] = lse_of(sm.m, l);
  // each lane's factor goes into its own row before the rows are staged
  const float inv = inv_of(l);
#pragma unroll
  for (int db = 0; db < NDB; ++db) sm.o[db] *= inv;
  store_rows<T, D>(lds + wave * AREA, sm.o, 1.f, lane, [&](int i) {
    return r0 + i < a.R ? row_ptr<T>(a.out, a.os, b, row_of(a, r0 + i, kvh)) : nullptr;
  });
}

// Few rows: a workgroup takes 32 rows, and its four waves go through the keys' tiles by
// turns, each with a ring of its own (no barrier until their sums are joined through
// LDS); the keys may be split over workgroups as well, a.per of them each, so that the
// splits of a long and a short batch element are of one size and those past its end do
// nothing. Bound by the states' bytes: 128 KiB per CU are in flight. One token of 16
// heads against 4096 states of 4, batch 16 of lengths 2048 to 4096 (50 MB): 13.7 us from
// memory (3.7 TB/s), 11.9 where the caches hold the states, and 4 to join.
template <typename T, int D>
struct FewRows {
  using Tl = Tile<T, D>;
  // (bf16: two workgroups per CU, at d = 64 with one stage per wave, 15.7 us against 17.3
  // with two and one workgroup; fp32 is seldom short of work per byte and keeps two)
  static constexpr int STAGE = 2 * BN * Tl::ROW, RING = 8 * STAGE <= (sizeof(T) == 2 ? 64 : 128) * 1024 ? 2 : 1;
  static constexpr int PER = (16 * Tl::NDB + 2) * 64 * 4;   // a wave's sums, maxima and O
  static constexpr int LDSB = 4 * RING * STAGE;
  static_assert(3 * PER + 32 * (Tl::ROW + 16) <= LDSB, "the waves' sums and the rows' staging must fit the rings");
  using Copy = KvCopy<T, D, 1>;
  static_assert(Copy::LPT < 64, "vmcnt range");
  const char *K, *V;
  uint32_t kr, vr;
  int k0, k1, nt;   // keys [k0, k1), this wave's tiles: wave, wave + 4, ...
  char *ring;
  __device__ __forceinline__ void init(const CrossArgs &a, char *lds, int sp, int b, int kvh, int wave) {
    const int len = keys_of(a, b);
    k0 = sp * a.per;
    k1 = min(k0 + a.per, len);
    const int tiles = k1 > k0 ? (k1 - k0 + BN - 1) / BN : 0;
    nt = (tiles - wave + 3) / 4;
    K = head_ptr(a.k, a.ks, b, kvh);
    V = head_ptr(a.v, a.vs, b, kvh);
    kr = a.ks.row * 16;
    vr = a.vs.row * 16;
    ring = lds + wave * RING * STAGE;
  }
  __device__ __forceinline__ int first(int i, int wave) const { return k0 + (4 * i + wave) * BN; }
  __device__ __forceinline__ void issue(int i, int wave, int lane) const {
    const int at = first(i, wave);
    Copy::issue(K + (int64_t)at * kr, V + (int64_t)at * vr, kr, vr, k1 - 1 - at, ring + (i % RING) * STAGE, 0, lane);
  }
  // f(stage, keys from its first on) for each of the wave's tiles
  template <class F>
  __device__ __forceinline__ void walk(int wave, int lane, F f) const {
    for (int i = 0; i < nt; ++i) {
      // (no barrier: the wave reads only what it copied itself)
      if (RING == 2 && i + 1 < nt) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(Copy::LPT) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      f(ring + (i % RING) * STAGE, k1 - first(i, wave));
      if (i + RING < nt) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // its reads of the stage are done
        issue(i + RING, wave, lane);
      }
    }
  }
  __device__ __forceinline__ void start(int wave, int lane) const {
#pragma unroll
    for (int i = 0; i < RING; ++i)
      if (i < nt) issue(i, wave, lane);
  }
};

template <typename T, int D>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) cross_fwd_few(CrossArgs a) {
  using Tl = Tile<T, D>;
  using Few = FewRows<T, D>;
  constexpr int NDB = Tl::NDB;
  __shared__ __attribute__((aligned(16))) char lds[Few::LDSB];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int logical = deal(blockIdx.x, a.unit);
  if (logical >= a.total) return;
  const int rt = logical % a.n_rtiles, t = logical / a.n_rtiles;
  const int sp = t % a.splits, bk = t / a.splits, b = bk / a.kv, kvh = bk - b * a.kv;
  Few few;
  few.init(a, lds, sp, b, kvh, wave);
  if (few.k0 >= few.k1 && a.splits > 1) return;
  few.start(wave, lane);
  const int r0 = rt * 32, r = r0 + col;
  typename Tl::Frag q;
  Tl::load(q, row_ptr<T>(a.q, a.qs, b, row_of(a, min(r, a.R - 1), kvh)), half);
  Tl tl;
  tl.init(lane);
  Softmax<T, D> sm;
  sm.init();
  few.walk(wave, lane, [&](const char *st, int left) {
    sm.tile(tl, st, st + BN * Tl::ROW, q, a.scale_log2, left, half);
  });
  const float m = sm.m;   // (no tile: -inf, and zeros)
  float l = sm.l + __shfl_xor(sm.l, 32);

  // Waves 1 to 3 hand over O, m and l.
  wait_then_barrier<0>();
  float *ex = reinterpret_cast<float *>(lds) + lane;
  auto at = [&](int w, int i) { return (w - 1) * (Few::PER / 4) + i * 64; };
  if (wave) {
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) ex[at(wave, 16 * db + v)] = sm.o[db][v];
    ex[at(wave, 16 * NDB)] = m;
    ex[at(wave, 16 * NDB + 1)] = l;
  }
  wait_then_barrier<0>();
  if (wave) return;
  float top = m;
#pragma unroll
  for (int w = 1; w < 4; ++w) top = fmaxf(top, ex[at(w, 16 * NDB)]);
  const float ref = top == -__builtin_inff() ? 0.f : top;
  {
    const float f = __builtin_amdgcn_exp2f(m - ref);
    l *= f;
#pragma unroll
    for (int db = 0; db < NDB; ++db) sm.o[db] *= f;
  }
#pragma unroll
  for (int w = 1; w < 4; ++w) {
    const float f = __builtin_amdgcn_exp2f(ex[at(w, 16 * NDB)] - ref);
    l += f * ex[at(w, 16 * NDB + 1)];
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) sm.o[db][v] = __builtin_fmaf(f, ex[at(w, 16 * db + v)], sm.o[db][v]);
  }
  if (a.splits > 1) {
    const int64_t to = ((int64_t)bk * a.splits + sp) * a.R + r;
    if (r < a.R) {
      float *p = a.part + to * D;
      Tl::columns(sm.o, half, [&](int c, f32x4 v) { *reinterpret_cast<f32x4 *>(p + c) = v; });
      if (half == 0) a.part_ml[to] = make_float2(top, l);
    }
    return;
  }
  if (a.lse && half == 0 && r < a.R) a.lse[(int64_t)bk * a.R + r] = lse_of(top, l);
  const float inv = inv_of(l);
#pragma unroll
  for (int db = 0; db < NDB; ++db) sm.o[db] *= inv;
  store_rows<T, D>(lds + 3 * Few::PER, sm.o, 1.f, lane, [&](int i) {
    return r0 + i < a.R ? row_ptr<T>(a.out, a.os, b, row_of(a, r0 + i, kvh)) : nullptr;
  });
}

// Up to 128 keys (a text's tokens): keys and values stay in LDS, and a workgroup's waves,
// each for itself, go through blocks of 32 rows with the next block's queries in flight.
// Bound by a block's latency: its loads, products and stores follow one another, with one
// block ahead and 1.5 waves per SIMD (vector issue 36%). 16 x 6 heads of 32, 4096 rows
// against 77 keys 19.3 us from memory (2.6 TB/s), 18.4 over one set of inputs (645 as
// elementary operations); 4 x 8 heads of 64, 16384 rows 39.5 (3.4 TB/s) and 35.8.
// Workgroups per CU of the kernels whose keys stay in LDS: what their registers (three,
// two for rows of 128 bytes) or LDS (fp32 rows of 64: 98 KiB, one) leave.
constexpr int short_waves(int row_bytes) { return row_bytes > 128 ? 1 : (row_bytes > 64 ? 2 : 3); }

template <typename T, int D>
__global__ void __launch_bounds__(256, short_waves(sizeof(T) * D)) cross_fwd_short(CrossArgs a) {
  using Tl = Tile<T, D>;
  constexpr int NDB = Tl::NDB, STAGE = 2 * BN * Tl::ROW, AREA = 32 * (Tl::ROW + 16);
  __shared__ __attribute__((aligned(16))) char lds[2 * STAGE + 4 * AREA];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int logical = deal(blockIdx.x, a.unit);
  if (logical >= a.total) return;
  const int part = logical % a.row_parts, bk = logical / a.row_parts, b = bk / a.kv, kvh = bk - b * a.kv;
  const int len = keys_of(a, b), nt = (len + BN - 1) / BN;
  const char *K = head_ptr(a.k, a.ks, b, kvh), *V = head_ptr(a.v, a.vs, b, kvh);
  const uint32_t kr = a.ks.row * 16, vr = a.vs.row * 16;
  for (int i = 0; i < nt; ++i)
    KvCopy<T, D, 4>::issue(K + (int64_t)i * BN * kr, V + (int64_t)i * BN * vr, kr, vr, len - 1 - i * BN, lds + i * STAGE, wave, lane);
  const int nblk = (a.R + 31) / 32, step = 4 * a.row_parts;
  int rb = part * 4 + wave;
  auto load = [&](typename Tl::Frag &q, int blk) {
    Tl::load(q, row_ptr<T>(a.q, a.qs, b, row_of(a, min(blk * 32 + col, a.R - 1), kvh)), half);
  };
  typename Tl::Frag q;
  if (rb < nblk) load(q, rb);
  Tl tl;
  tl.init(lane);
  wait_vmem_all();
  wait_then_barrier<0>();
  for (; rb < nblk; rb += step) {
    typename Tl::Frag next;
    load(next, min(rb + step, nblk - 1));
    Softmax<T, D> sm;
    sm.init();
    for (int i = 0; i < nt; ++i) {
      const char *st = lds + i * STAGE;
      sm.tile(tl, st, st + BN * Tl::ROW, q, a.scale_log2, len - i * BN, half);
    }
    const float l = sm.l + __shfl_xor(sm.l, 32), inv = inv_of(l);
    const int r0 = rb * 32;
    if (a.lse && half == 0 && r0 + col < a.R) a.lse[(int64_t)bk * a.R + r0 + col] = lse_of(sm.m, l);
#pragma unroll
    for (int db = 0; db < NDB; ++db) sm.o[db] *= inv;
    store_rows<T, D>(lds + 2 * STAGE + wave * AREA, sm.o, 1.f, lane, [&](int i) {
      return r0 + i < a.R ? row_ptr<T>(a.out, a.os, b, row_of(a, r0 + i, kvh)) : nullptr;
    });
#pragma unroll
    for (int c = 0; c < Tl::NCH; ++c) q[c] = next[c];
  }
}

// Joins the partial sums of the key splits. One wave per row: D / 4 lanes take four
// columns each, 256 / D groups of them every 256 / D-th split.
template <typename T, int D>
__global__ void __launch_bounds__(256) cross_join(CrossArgs a) {
  constexpr int TPR = D / 4, SL = 64 / TPR;
  const int lane = threadIdx.x & 63, c = lane % TPR * 4, first = lane / TPR;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= (int64_t)a.B * a.kv * a.R) return;
  const int bk = (int)(row / a.R), r = (int)(row - (int64_t)bk * a.R), b = bk / a.kv, kvh = bk - b * a.kv;
  const int n = (keys_of(a, b) + a.per - 1) / a.per;   // splits with keys
  const float2 *ml = a.part_ml + (int64_t)bk * a.splits * a.R + r;
  const float *p = a.part + ((int64_t)bk * a.splits * a.R + r) * D + c;
  float m = -__builtin_inff();
#pragma unroll 4
  for (int s = first; s < n; s += SL) m = fmaxf(m, ml[(int64_t)s * a.R].x);
#pragma unroll
  for (int x = TPR; x < 64; x *= 2) m = fmaxf(m, __shfl_xor(m, x));
  const float ref = m == -__builtin_inff() ? 0.f : m;
  float l = 0.f;
  f32x4 o = {};
#pragma unroll 4
  for (int s = first; s < n; s += SL) {
    const float2 e = ml[(int64_t)s * a.R];
    const f32x4 x = *reinterpret_cast<const f32x4 *>(p + (int64_t)s * a.R * D);
    const float w = __builtin_amdgcn_exp2f(e.x - ref);
    l += w * e.y;
    o += w * x;
  }
#pragma unroll
  for (int x = TPR; x < 64; x *= 2) {
    l += __shfl_xor(l, x);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], x);
  }
  if (first) return;
  if (a.lse && c == 0) a.lse[(int64_t)bk * a.R + r] = lse_of(m, l);
  put4<T>(row_ptr<T>(a.out, a.os, b, row_of(a, r, kvh)) + c, o * inv_of(l));
}

// A wave's 32 rows of the backward: q, dout and the statistics.
template <typename T, int D>
struct BwdRows {
  using Tl = Tile<T, D>;
  typename Tl::Frag q, g, out;
  float lraw, lse2, ndelta;
  __device__ __forceinline__ void load(const CrossArgs &a, int bk, int b, int kvh, int r, int half) {
    const int rc = min(r, a.R - 1);   // (rows past the last read it and store nothing)
    const Row rw = row_of(a, rc, kvh);
    Tl::load(q, row_ptr<T>(a.q, a.qs, b, rw), half);
    Tl::load(g, row_ptr<T>(a.dout, a.gs, b, rw), half);
    Tl::load(out, row_ptr<T>(a.out, a.os, b, rw), half);
    lraw = a.lse[(int64_t)bk * a.R + rc];
  }
  // The statistics: lse log2 e (+inf for a row without a key and for the padding of the
  // last tile, which makes every weight exp2(s - inf) = 0) and -delta.
  __device__ __forceinline__ void finish(const CrossArgs &a, int r) {
    const float d = Tl::dot(out, g);
    ndelta = -(d + __shfl_xor(d, 32));
    lse2 = r < a.R && lraw != -__builtin_inff() ? lraw * kLog2e : __builtin_inff();
  }
  // ... stored for the dk / dv kernel.
  __device__ __forceinline__ void keep(const CrossArgs &a, int bk, int r, int half) const {
    if (half) return;
    const int64_t at = (int64_t)bk * a.Rp + r;
    a.stats[at] = lse2;
    a.stats[(int64_t)a.B * a.kv * a.Rp + at] = ndelta;
  }
  // bf16: <dout, out> takes the rounding of out into delta, for all keys alike, and
  // where few keys share a row's weight, dS = P (dP - delta) cancels and is left with
  // it (dq and dk of 3 and 20 keys 3.1e-3 off in the 2-norm instead of 2.3e-3, of one to
  // three keys 4.4e-3). As the weights sum to 1, the sum of a row's dS is just what its
  // delta lacks. Where a row may see few keys the sum `excess` is taken along, and
  //   dq = scale (sum_j dS_j k_j - excess sum_j P_j k_j),
  // the second product beside the first; delta is put right for dk.
  static constexpr bool kMends = sizeof(T) == 2;
  struct Sums {
    f32x16 ds[Tl::NDB], p[Tl::NDB];
    float excess;
    __device__ __forceinline__ void init() {
#pragma unroll
      for (int db = 0; db < Tl::NDB; ++db) ds[db] = p[db] = f32x16{};
      excess = 0.f;
    }
  };
  // Sums over the `left` keys of a tile (K tile, then V tile, at st).
  // MEND: with the excess and the second product. DRY: the excess alone.
  template <bool MEND, bool DRY = false>
  __device__ __forceinline__ void tile(const Tl &tl, const char *st, float scale, int left, int half, Sums &sum) const {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      if (32 * kb >= left) break;
      const char *blk = st + kb * 32 * Tl::ROW;
      f32x16 s, dp;
      tl.rows_times(blk, q, s);
      tl.rows_times(blk + BN * Tl::ROW, g, dp);
      if (left < 32 * kb + 32) mask_tail(s, left - 32 * kb, half);
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[v], scale, -lse2));
        s[v] = p * (dp[v] + ndelta);
        if (MEND || DRY) sum.excess += s[v];
        dp[v] = p;
      }
      if (!DRY) tl.cols_times(blk, s, sum.ds);
      if (MEND) tl.cols_times(blk, dp, sum.p);
    }
  }
  // The row's whole excess (half: this lane's part of it) into delta and the sums.
  template <bool MEND>
  __device__ __forceinline__ void mend(Sums &sum) {
    const float excess = sum.excess + __shfl_xor(sum.excess, 32);
    ndelta -= excess;
    if (MEND) {
#pragma unroll
      for (int db = 0; db < Tl::NDB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) sum.ds[db][v] = __builtin_fmaf(-excess, sum.p[db][v], sum.ds[db][v]);
    }
  }
};

// Keys up to which cross_dq mends delta, in a pass of its own (it has no registers for
// the second product). Beyond, the rounding of out is below 3% of the result's error.
constexpr int kMendKeys = 256;

// dq, and the rows' statistics for the next kernel. Many rows: as cross_fwd.
template <typename T, int D>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 3 : 2) cross_dq(CrossArgs a) {
  using Tl = Tile<T, D>;
  constexpr int NDB = Tl::NDB, RING = fwd_ring<T, D>(), NW = 4;
  constexpr int STAGE = 2 * BN * Tl::ROW;
  constexpr int AREA = 32 * (Tl::ROW + 16);
  using Copy = KvCopy<T, D, NW>;
  __shared__ __attribute__((aligned(16))) char lds[RING * STAGE];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int logical = deal(blockIdx.x, a.unit);
  if (logical >= a.total) return;
  const int rt = logical % a.n_rtiles, bk = logical / a.n_rtiles, b = bk / a.kv, kvh = bk - b * a.kv;
  const int len = keys_of(a, b), nt = (len + BN - 1) / BN;
  const char *K = head_ptr(a.k, a.ks, b, kvh), *V = head_ptr(a.v, a.vs, b, kvh);
  const uint32_t kr = a.ks.row * 16, vr = a.vs.row * 16;
  auto issue = [&](int i) {
    const int at = i * BN;
    Copy::issue(K + (int64_t)at * kr, V + (int64_t)at * vr, kr, vr, len - 1 - at, lds + (i % RING) * STAGE, wave, lane);
  };
  const int r0 = (rt * NW + wave) * 32;
  BwdRows<T, D> rows;
  Tl tl;
  tl.init(lane);
  typename BwdRows<T, D>::Sums sum;
  sum.init();
  auto start = [&]() {
#pragma unroll
    for (int i = 0; i < RING - 1; ++i)
      if (i < nt) issue(i);
  };
  auto walk = [&](auto f) __attribute__((always_inline)) {
    for (int i = 0; i < nt; ++i) {
      wait_tiles_then_barrier<Copy::LPT, RING - 2>(min(RING - 2, nt - 1 - i));
      if (i + RING - 1 < nt) issue(i + RING - 1);
      f(lds + (i % RING) * STAGE, len - i * BN);
    }
    wait_then_barrier<0>();   // every wave is done with the ring
  };
  start();
  rows.load(a, bk, b, kvh, r0 + col, half);
  wait_vmem_all();
  rows.finish(a, r0 + col);
  if (rows.kMends && len <= kMendKeys) {
    walk([&](const char *st, int left) { rows.template tile<false, true>(tl, st, a.scale_log2, left, half, sum); });
    rows.template mend<false>(sum);
    start();
  }
  walk([&](const char *st, int left) { rows.template tile<false>(tl, st, a.scale_log2, left, half, sum); });
  rows.keep(a, bk, r0 + col, half);
  store_rows<T, D>(lds + wave * AREA, sum.ds, a.scale, lane, [&](int i) {
    return r0 + i < a.R ? row_ptr<T>(a.dq, a.dqs, b, row_of(a, r0 + i, kvh)) : nullptr;
  });
}

// Few rows: as cross_fwd_few.
template <typename T, int D>
__global__ void __launch_bounds__(256, sizeof(T) * D <= 64 ? 2 : 1) cross_dq_few(CrossArgs a) {
  using Tl = Tile<T, D>;
  using Few = FewRows<T, D>;
  constexpr int NDB = Tl::NDB;
  __shared__ __attribute__((aligned(16))) char lds[Few::LDSB];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int logical = deal(blockIdx.x, a.unit);
  if (logical >= a.total) return;
  const int rt = logical % a.n_rtiles, bk = logical / a.n_rtiles, b = bk / a.kv, kvh = bk - b * a.kv;
  Few few;
  few.init(a, lds, 0, b, kvh, wave);
  few.start(wave, lane);
  const int r0 = rt * 32;
  BwdRows<T, D> rows;
  rows.load(a, bk, b, kvh, r0 + col, half);
  rows.finish(a, r0 + col);
  Tl tl;
  tl.init(lane);
  constexpr bool MEND = BwdRows<T, D>::kMends;
  constexpr int PER = ((MEND ? 2 : 1) * 16 * NDB + 1) * 64;   // floats that a wave hands over
  static_assert(3 * PER * 4 + 32 * (Tl::ROW + 16) <= Few::LDSB, "the waves' sums and the rows' staging must fit the rings");
  typename BwdRows<T, D>::Sums sum;
  sum.init();
  few.walk(wave, lane, [&](const char *st, int left) { rows.template tile<MEND>(tl, st, a.scale_log2, left, half, sum); });
  wait_then_barrier<0>();
  float *ex = reinterpret_cast<float *>(lds) + lane;
  auto at = [&](int w, int i) { return (w - 1) * PER + i * 64; };
  if (wave) {
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        ex[at(wave, 16 * db + v)] = sum.ds[db][v];
        if (MEND) ex[at(wave, 16 * (NDB + db) + v)] = sum.p[db][v];
      }
    ex[at(wave, PER / 64 - 1)] = sum.excess;
  }
  wait_then_barrier<0>();
  if (wave) return;
#pragma unroll
  for (int w = 1; w < 4; ++w) {
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        sum.ds[db][v] += ex[at(w, 16 * db + v)];
        if (MEND) sum.p[db][v] += ex[at(w, 16 * (NDB + db) + v)];
      }
    sum.excess += ex[at(w, PER / 64 - 1)];
  }
  if (MEND) rows.template mend<true>(sum);
  rows.keep(a, bk, r0 + col, half);
  store_rows<T, D>(lds + 3 * PER * 4, sum.ds, a.scale, lane, [&](int i) {
    return r0 + i < a.R ? row_ptr<T>(a.dq, a.dqs, b, row_of(a, r0 + i, kvh)) : nullptr;
  });
}

// The same for up to 128 keys, which stay in LDS: as cross_fwd_short, with the next
// block's q, dout, out and lse in flight.
template <typename T, int D>
__global__ void __launch_bounds__(256, short_waves(sizeof(T) * D)) cross_dq_short(CrossArgs a) {
  using Tl = Tile<T, D>;
  constexpr int NDB = Tl::NDB, STAGE = 2 * BN * Tl::ROW, AREA = 32 * (Tl::ROW + 16);
  __shared__ __attribute__((aligned(16))) char lds[2 * STAGE + 4 * AREA];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int logical = deal(blockIdx.x, a.unit);
  if (logical >= a.total) return;
  const int part = logical % a.row_parts, bk = logical / a.row_parts, b = bk / a.kv, kvh = bk - b * a.kv;
  const int len = keys_of(a, b), nt = (len + BN - 1) / BN;
  const char *K = head_ptr(a.k, a.ks, b, kvh), *V = head_ptr(a.v, a.vs, b, kvh);
  const uint32_t kr = a.ks.row * 16, vr = a.vs.row * 16;
  for (int i = 0; i < nt; ++i)
    KvCopy<T, D, 4>::issue(K + (int64_t)i * BN * kr, V + (int64_t)i * BN * vr, kr, vr, len - 1 - i * BN, lds + i * STAGE, wave, lane);
  // (blocks up to the padded end of the list: their statistics are read by the next kernel)
  const int nblk = a.Rp / 32, step = 4 * a.row_parts;
  int rb = part * 4 + wave;
  BwdRows<T, D> rows;
  rows.load(a, bk, b, kvh, min(rb, nblk - 1) * 32 + col, half);
  Tl tl;
  tl.init(lane);
  wait_vmem_all();
  wait_then_barrier<0>();
  for (; rb < nblk; rb += step) {
    const int r0 = rb * 32;
    rows.finish(a, r0 + col);
    BwdRows<T, D> next;
    next.load(a, bk, b, kvh, min(rb + step, nblk - 1) * 32 + col, half);
    constexpr bool MEND = BwdRows<T, D>::kMends;
    typename BwdRows<T, D>::Sums sum;
    sum.init();
    for (int i = 0; i < nt; ++i) rows.template tile<MEND>(tl, lds + i * STAGE, a.scale_log2, len - i * BN, half, sum);
    if (MEND) rows.template mend<true>(sum);
    rows.keep(a, bk, r0 + col, half);
    store_rows<T, D>(lds + 2 * STAGE + wave * AREA, sum.ds, a.scale, lane, [&](int i) {
      return r0 + i < a.R ? row_ptr<T>(a.dq, a.dqs, b, row_of(a, r0 + i, kvh)) : nullptr;
    });
    rows = next;
  }
}

// How dk and dv are shared out over a.pieces workgroups (0: one to a key tile): the tiles
// that hold seen keys, of which only the device knows the number, get as many row splits
// as make that many workgroups. (Two elements, 4 heads' rows of 4096 against 1000 of 4096
// keys: 46 us, 138 with the splits of 4096.) a.uneven = 0: there are as many as the rows
// allow anyway, no lengths, or over 64 elements, and all keys count as seen.
struct KeyTiles {
  int all;             // of all batch elements and key heads
  int before, of;      // before and of batch element `lane`
};
__device__ __forceinline__ int tiles_of(const CrossArgs &a, int len) { return (len + (1 << a.kshift) - 1) >> a.kshift; }
__device__ __forceinline__ KeyTiles key_tiles(const CrossArgs &a, int lane) {
  const int n = lane < a.B ? tiles_of(a, keys_of(a, lane)) * a.kv : 0;
  int sum = n;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(sum, o);
    if (lane >= o) sum += x;
  }
  return {__builtin_amdgcn_readlane(sum, 63), sum - n, n};
}
__device__ __forceinline__ int splits_of(const CrossArgs &a, int tiles) {
  return clampi(a.pieces / max(tiles, 1), 1, a.splits);
}

// dk and dv of KB blocks of 32 keys: wave w takes the keys of block w % KB against half
// w / KB of the rows of every step (RB blocks of 32 each). Rows come into an LDS ring by
// the 16-byte DMA; the halves are added through LDS at the end. Bound by the waves' vector
// and matrix work, two waves per SIMD (200 registers): 4096 rows of 8 heads on 2 against
// 4096 keys, batch 2, heads of 64 in bf16: 139 to 153 us (900 to 990 TFLOP/s); with 64 keys
// to a workgroup, and twice the rows' traffic, the whole backward takes 13 us longer.
template <typename T, int D, int KB, int RB>
__global__ void __launch_bounds__(128 * KB, 2) cross_dkdv(CrossArgs a) {
  using Tl = Tile<T, D>;
  constexpr int NDB = Tl::NDB, NW = 2 * KB, BR = 64 * RB;   // waves, rows per step
  constexpr int TILE = BR * Tl::ROW;
  constexpr int STAT = 2 * TILE, STAGE = STAT + BR * 8;
  constexpr int CPW = BR * Tl::CPR / (64 * NW);
  constexpr int RING = NW == 8 && 3 * STAGE <= 160 * 1024 ? 3 : 2;
  constexpr int SW = BR * 2 / 64;                  // waves that copy statistics
  constexpr int LPT = 2 * CPW + 1;
  constexpr int AREA = 32 * (Tl::ROW + 16);
  constexpr int XCH = KB * 2 * NDB * 16 * 64 * 4;
  constexpr int LDSB = RING * STAGE < XCH ? XCH : RING * STAGE;
  static_assert(NW * AREA <= LDSB && SW <= NW, "staging, statistics");
  static_assert(BR * Tl::CPR % (64 * NW) == 0, "copies must split evenly");
  __shared__ __attribute__((aligned(16))) char lds[LDSB];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5, kb = wave % KB, rh = wave / KB;
  const int logical = deal(blockIdx.x, a.unit);
  if (logical >= a.total) return;
  // Workgroups go by (batch, key head, split, tile): those side by side share their rows.
  int splits = 1, per_head = a.n_ktiles, b = 0, in = logical;
  if (a.uneven) {
    const KeyTiles kt = key_tiles(a, lane);
    splits = splits_of(a, kt.all);
    const uint64_t hit = __ballot(kt.before * splits <= logical && logical < (kt.before + kt.of) * splits);
    if (!hit) return;
    b = (int)__builtin_ctzll(hit);
    in -= __builtin_amdgcn_readlane(kt.before, b) * splits;
    per_head = __builtin_amdgcn_readlane(kt.of, b) / a.kv;
  } else {
    if (a.pieces) splits = splits_of(a, a.B * a.kv * per_head);
    b = logical / (a.kv * splits * per_head);
    if (b >= a.B) return;
    in -= b * a.kv * splits * per_head;
  }
  const int t = in / per_head, kt = in - t * per_head, kvh = t / splits, sp = t - kvh * splits, bk = b * a.kv + kvh;
  const int len = keys_of(a, b);
  const int j0 = (kt * KB + kb) * 32, kpos = j0 + col;   // this wave's first key, this lane's

  // (no key of the tile is seen: zeros, which the joining launch knows by itself)
  if (a.pieces && kt * KB * 32 >= len) return;

  // This split's rows: whole steps.
  const int steps = (a.R + BR - 1) / BR, per = (steps + splits - 1) / splits;
  const int i0 = min(sp * per, steps), i1 = kt * KB * 32 < len ? min(i0 + per, steps) : i0;
  const float *S = a.stats + (int64_t)bk * a.Rp;
  const int64_t dofs = (int64_t)a.B * a.kv * a.Rp;   // from lse to -delta
  auto issue = [&](int i) {
    char *stage = lds + (i - i0) % RING * STAGE;
#pragma unroll
    for (int j = 0; j < CPW; ++j) {
      const int p = (j * NW + wave) * 64 + lane, rr = p / Tl::CPR, c = (p % Tl::CPR) ^ Tl::swz(rr);
      // (rows past the last read it; their statistics make their weights 0)
      const Row rw = row_of(a, min(i * BR + rr, a.R - 1), kvh);
      lds_dma16(reinterpret_cast<const char *>(row_ptr<T>(a.q, a.qs, b, rw)) + c * 16, lds_addr(stage + (j * NW + wave) * 1024));
      lds_dma16(reinterpret_cast<const char *>(row_ptr<T>(a.dout, a.gs, b, rw)) + c * 16,
                lds_addr(stage + TILE + (j * NW + wave) * 1024));
    }
    // 64 rows' lse, or -delta, per wave (the waves past them copy the last again, so that
    // all have the same number in flight)
    const int w = min(wave, SW - 1), which = w / (SW / 2), part = w % (SW / 2);
    lds_dma4(S + which * dofs + i * BR + part * 64 + lane, lds_addr(stage + STAT + which * BR * 4 + part * 256));
  };
#pragma unroll
  for (int i = 0; i < RING - 1; ++i)
    if (i0 + i < i1) issue(i0 + i);

  const Row krow = {(uint32_t)kvh, (uint32_t)min(kpos, max(len - 1, 0))};   // (unseen keys: not stored)
  typename Tl::Frag k, v;
  Tl::load(k, row_ptr<T>(a.k, a.ks, b, krow), half);
  Tl::load(v, row_ptr<T>(a.v, a.vs, b, krow), half);
  Tl tl;
  tl.init(lane);
  f32x16 dk[NDB], dv[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) dk[db] = dv[db] = f32x16{};
  wait_vmem_all();

  for (int i = i0; i < i1; ++i) {
    wait_tiles_then_barrier<LPT, RING - 2>(min(RING - 2, i1 - 1 - i));
    if (i + RING - 1 < i1) issue(i + RING - 1);
    if (j0 >= len) continue;   // (none of the wave's keys is seen)
    const char *st = lds + (i - i0) % RING * STAGE;
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

  // Half 1 hands its dk to half 0, which hands it its dv; then each holds one sum.
  wait_then_barrier<0>();   // every wave is done with the ring
  float *xch = reinterpret_cast<float *>(lds);
  auto at = [&](int which, int db, int e) { return (((kb * 2 + which) * NDB + db) * 16 + e) * 64 + lane; };
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) xch[at(rh, db, e)] = rh ? dk[db][e] : dv[db][e];
  wait_then_barrier<0>();
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) dk[db][e] = (rh ? dv[db][e] : dk[db][e]) + xch[at(1 - rh, db, e)];
  wait_then_barrier<0>();
  if (a.pieces) {
    if (kpos < len) {
      float *p = a.part + (((int64_t)logical * (32 * KB) + 32 * kb + col) * 2 + rh) * D;
      Tl::columns(dk, half, [&](int c, f32x4 x) { *reinterpret_cast<f32x4 *>(p + c) = x; });
    }
    return;
  }
  if (kpos >= len) {
#pragma unroll
    for (int db = 0; db < NDB; ++db) dk[db] = f32x16{};
  }
  const CrossStride &os = rh ? a.dvs : a.dks;
  store_rows<T, D>(lds + wave * AREA, dk, rh ? 1.f : a.scale, lane, [&](int i) {
    return j0 + i < a.M ? row_ptr<T>(rh ? a.dv : a.dk, os, b, {(uint32_t)kvh, (uint32_t)(j0 + i)}) : nullptr;
  });
}

// Adds the partial sums of the row splits: one thread per key, gradient and four columns,
// or a.ways of them where there are few keys of many splits, added through LDS in order.
template <typename T, int D>
__global__ void __launch_bounds__(256) cross_sum(CrossArgs a) {
  constexpr int TPR = D / 4;
  __shared__ f32x4 lds[256];
  const int lanes = 256 / a.ways, way = (int)threadIdx.x / lanes, slot = (int)threadIdx.x - way * lanes;
  const int64_t idx = (int64_t)blockIdx.x * lanes + slot, keys = (int64_t)a.B * a.kv * a.M;
  const int c = (int)(idx % TPR) * 4, which = (int)(idx / TPR % 2);
  const int64_t key = min(idx / (2 * TPR), keys - 1);   // (every lane takes part in the scan)
  const int bk = (int)(key / a.M), j = (int)(key - (int64_t)bk * a.M), b = bk / a.kv, kvh = bk - b * a.kv;
  int tiles = a.B * a.kv * a.n_ktiles, per_head = a.n_ktiles, before = b * a.kv * a.n_ktiles;
  const int len = keys_of(a, b);
  if (a.uneven) {
    const KeyTiles kt = key_tiles(a, threadIdx.x & 63);
    tiles = kt.all;
    per_head = tiles_of(a, len);
    before = __shfl(kt.before, b);
  }
  f32x4 sum = {};
  if (j < len) {
    const int splits = splits_of(a, tiles), piece = (before + kvh * per_head) * splits + (j >> a.kshift);
    const float *p = a.part + ((((int64_t)piece << a.kshift) + (j & ((1 << a.kshift) - 1))) * 2 + which) * D + c;
    const int64_t step = ((int64_t)per_head << a.kshift) * 2 * D;
#pragma unroll 8
    for (int s = way; s < splits; s += a.ways) sum += *reinterpret_cast<const f32x4 *>(p + s * step);
  }
  if (a.ways > 1) {
    lds[threadIdx.x] = sum;
    __syncthreads();
    if (way == 0)
      for (int k = 1; k < a.ways; ++k) sum += lds[slot + k * lanes];
  }
  if (way || idx / (2 * TPR) >= keys) return;
  const CrossStride &os = which ? a.dvs : a.dks;
  T *dst = row_ptr<T>(which ? a.dv : a.dk, os, b, {(uint32_t)kvh, (uint32_t)j});
  put4<T>(dst + c, sum * (which ? 1.f : a.scale));
}

// Tiles of 32 rows, the keys shared by the waves, where tiles of 128 would leave CUs
// without work.
bool few_rows(const CrossArgs &a) { return (int64_t)a.B * a.kv * ((a.R + 127) / 128) < device_cu_count(); }

// Keys that stay in LDS, against rows enough that they are met more than once.
bool keys_stay(const CrossArgs &a) { return a.M <= 128 && a.R > 32; }

// Blocks of 32 keys of a dk / dv workgroup: four (eight waves, one workgroup per CU)
// where those fill the CUs, runs of 128 rows included; two, of four waves, otherwise.
int kv_blocks(const CrossArgs &a) {
  const int64_t most = (int64_t)a.B * a.kv * ((a.M + 127) / 128) * ((a.R + 127) / 128);
  return a.M > 64 && most >= device_cu_count() ? 4 : 2;
}

// Grid of `total` pieces of work, dealt to the XCDs in runs.
dim3 deal_grid(CrossArgs &a, int64_t total) {
  a.total = (int32_t)total;
  a.unit = (int32_t)std::max<int64_t>(1, std::min<int64_t>(32, total / 32));
  const int64_t round = 8 * a.unit;
  return dim3((uint32_t)((total + round - 1) / round * round));
}

template <typename T, int D>
hipError_t fwd(CrossArgs &a, hipStream_t s) {
  const int64_t bk = (int64_t)a.B * a.kv;
  if (keys_stay(a)) {
    const dim3 grid = deal_grid(a, bk * a.row_parts);
    hipLaunchKernelGGL((cross_fwd_short<T, D>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
  }
  if (!few_rows(a)) {
    a.n_rtiles = (a.R + 127) / 128;
    const dim3 grid = deal_grid(a, bk * a.n_rtiles);
    hipLaunchKernelGGL((cross_fwd<T, D>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
  }
  a.n_rtiles = (a.R + 31) / 32;
  const dim3 grid = deal_grid(a, bk * a.n_rtiles * a.splits);
  hipLaunchKernelGGL((cross_fwd_few<T, D>), grid, dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  hipLaunchKernelGGL((cross_join<T, D>), dim3((uint32_t)((bk * a.R + 3) / 4)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t bwd(CrossArgs &a, hipStream_t s) {
  constexpr int RB = sizeof(T) == 4 ? 1 : 2;
  const int64_t bk = (int64_t)a.B * a.kv;
  if (keys_stay(a)) {
    const dim3 grid = deal_grid(a, bk * a.row_parts);
    hipLaunchKernelGGL((cross_dq_short<T, D>), grid, dim3(256), 0, s, a);
  } else if (few_rows(a)) {
    a.n_rtiles = a.Rp / 32;   // (the padded rows' statistics as well)
    const dim3 grid = deal_grid(a, bk * a.n_rtiles);
    hipLaunchKernelGGL((cross_dq_few<T, D>), grid, dim3(256), 0, s, a);
  } else {
    a.n_rtiles = a.Rp / 128;
    const dim3 grid = deal_grid(a, bk * a.n_rtiles);
    hipLaunchKernelGGL((cross_dq<T, D>), grid, dim3(256), 0, s, a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  a.uneven = a.lengths && a.B <= 64 && a.pieces && a.pieces < bk * a.n_ktiles * a.splits;
  const dim3 grid = deal_grid(a, a.pieces ? a.pieces : bk * a.n_ktiles);
  if (a.kshift == 6) hipLaunchKernelGGL((cross_dkdv<T, D, 2, RB>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((cross_dkdv<T, D, 4, RB>), grid, dim3(512), 0, s, a);
  e = hipGetLastError();
  if (e != hipSuccess || !a.pieces) return e;
  const int64_t n = bk * a.M * 2 * (D / 4);
  a.ways = 1;
  while (a.ways < 16 && a.pieces / (bk * a.n_ktiles) >= 16 * a.ways && n * a.ways < 256 * (int64_t)device_cu_count()) a.ways *= 2;
  const int lanes = 256 / a.ways;
  hipLaunchKernelGGL((cross_sum<T, D>), dim3((uint32_t)((n + lanes - 1) / lanes)), dim3(256), 0, s, a);
  return hipGetLastError();
}

int up_to(int64_t want, int64_t most) { return (int)std::max<int64_t>(1, std::min(want, most)); }

}  // namespace

// How the rows are shared out where the keys stay in LDS: as many blocks to a wave as let
// all workgroups run at once.
static void share_rows(CrossArgs &a, int row_bytes) {
  const int64_t slots = (int64_t)device_cu_count() * short_waves(row_bytes), bk = (int64_t)a.B * a.kv;
  const int64_t parts = up_to(slots / bk, (a.R + 127) / 128), blocks = (a.R + 31) / 32;
  const int64_t each = (blocks + 4 * parts - 1) / (4 * parts);
  a.row_parts = (int)((blocks + 4 * each - 1) / (4 * each));
}

// Key splits of the forward: two workgroups per CU (their LDS fills it), of at least
// eight tiles each.
bool cross_fwd_plan(CrossArgs &a, int row_bytes) {
  a.splits = 1;
  a.per = (a.M + BN - 1) / BN * BN;
  share_rows(a, row_bytes);
  if (keys_stay(a) || !few_rows(a)) return false;
  const int64_t wgs = (int64_t)a.B * a.kv * ((a.R + 31) / 32), tiles = (a.M + BN - 1) / BN;
  const int splits = up_to(2 * device_cu_count() / wgs, (tiles + 7) / 8);
  a.per = (int)((tiles + splits - 1) / splits) * BN;
  a.splits = (a.M + a.per - 1) / a.per;
  return a.splits > 1;
}

// dk and dv: eight waves per CU where key tiles alone would leave half of the CUs without
// work, of at least 128 rows each. (Only the device knows the lengths, and so the splits.)
// Up to 512 rows in bf16 one workgroup takes them all: four steps cost no more than a
// launch that joins parts (512 rows, 6 heads of 64, 200 keys: the host issues the backward
// in 20 us, not 23, and a graph runs it in 17.9, not 18.4; 500 rows in fp32: 55, not 33).
// Rows of 64 bytes leave registers for sixteen waves, which pays from 1024 rows each on
// (132 tiles of 128 keys, 6144 rows, heads of 32: the backward 122 -> 91 us; 36 tiles, 4096
// rows: 31 against 34).
bool cross_bwd_plan(CrossArgs &a, int d, int es) {
  const int row_bytes = d * es;
  a.per = (a.M + BN - 1) / BN * BN;
  share_rows(a, row_bytes);
  const int kb = kv_blocks(a);
  a.kshift = kb == 2 ? 6 : 7;
  a.n_ktiles = (a.M + 32 * kb - 1) / (32 * kb);
  a.splits = (a.R + 127) / 128;
  const int64_t cus = device_cu_count(), tiles = (int64_t)a.B * a.kv * a.n_ktiles;
  const bool two = kb == 2 || (row_bytes <= 64 && tiles * a.R >= 2048 * cus);
  const int64_t slots = two ? 2 * cus : cus;
  a.pieces = a.R > (es == 2 ? 512 : 128) && 2 * tiles <= slots ? (int)std::min(slots, tiles * a.splits) : 0;
  return a.pieces > 0;
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
