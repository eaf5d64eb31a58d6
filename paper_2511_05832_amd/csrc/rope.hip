// Rotary positions (hla_rope): every pair (x1, x2) of a row's first `rot` features is
// turned by the angle a = position * frequency,
//   y1 = m (x1 cos a - x2 sin a),   y2 = m (x2 cos a + x1 sin a),
// with -a in place of a for the way back of a gradient; the other features are copied.
//
// Bound by HBM: each row is read and written once. A thread owns one unit of a row -
// the pairs of a 16-byte access or two, or features to copy - at one position, computes the
// unit's sines and cosines once, and goes through a run of (batch, head) slices with
// them, so the trigonometry (about 60 operations per pair) is shared. The runs leave the
// chip 32 waves per CU, two slices' loads in flight each. Measured, from memory / over one
// set of inputs, which the caches hold in part: 64x64 layer, 6 heads of 32, batch 16, bf16
// 23.6 / 18.0 us (4.3 / 5.6 TB/s); 65536 tokens, 8 + 2 heads of 64, fp32 63.5 / 51.4 us (5.3 /
// 6.5 TB/s; a copy of 1 GiB 5.1).
// Results go past the caches where a call moves more than they hold (256 MB; the fp32
// case 65.9 -> 64.7 us, the units' kernel 77 -> 70), while at 84 MB 16.4 -> 18.4 and the
// next kernel would find its inputs in memory.
//
// The angle is formed in float64 and reduced to a fraction of a turn before it is
// rounded: at position 10^5 and frequency 1 the float32 product is already 4e-3 off,
// while this is below 2e-7 up to 2^28.
#include <algorithm>

#include "attn_common.h"

namespace hla {
namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 2;   // slices whose loads are in flight together

// cos and sin (times the magnitude, the sign of the direction included) of position
// coordinate c and frequency f.
__device__ __forceinline__ void turn_of(double c, double f, const RopeArgs &p, float &cs, float &sn) {
  const double turns = c * f * 0.15915494309189535;   // 1 / 2 pi
  const float x = (float)(2.0 * (turns - rint(turns)));
  float s, co;
  sincospif(x, &s, &co);
  cs = co * p.magnitude;
  sn = s * (p.inverse ? -p.magnitude : p.magnitude);
}

// x c + y s, y the pair's other member. The order of roundings is written out, so that a row
// has the same bits in every kernel and in a call of any size.
__device__ __forceinline__ float turned(float x, float y, float c, float s) { return __builtin_fmaf(x, c, y * s); }

// The run of slices that a thread goes through with its sines and cosines: slice s is head
// s % HT of batch element s / HT (q's heads first, then k's). Per-batch positions: a group
// lies in one batch element.
struct Slices {
  int s0, s1, b, h, HT;
  __device__ __forceinline__ Slices(const RopeArgs &p, uint32_t grp) {
    HT = p.heads[0] + p.heads[1];
    if (p.pos_stride) {
      b = (int)(grp / (uint32_t)p.groups);
      const int g = (int)grp - b * p.groups;
      s0 = b * HT + g * p.run;
      s1 = min(s0 + p.run, (b + 1) * HT);
    } else {
      s0 = (int)grp * p.run;
      s1 = min(s0 + p.run, p.B * HT);
      b = s0 / HT;
    }
    h = s0 - b * HT;
  }
  // Row n's position, as (row, column) on a grid.
  __device__ __forceinline__ void position(const RopeArgs &p, int n, int &r, int &c) const {
    r = p.pos ? p.pos[(int64_t)(p.pos_stride ? b : 0) * p.pos_stride + n] : n;
    c = 0;
    if (p.axes == 2) {
      const int pos = r;
      r = (int)((uint32_t)pos / (uint32_t)p.grid_w);
      c = pos - r * p.grid_w;
    }
  }
  // Row n of the next m slices.
  template <typename T>
  __device__ __forceinline__ void rows(const RopeArgs &p, int m, int n, const T *(&src)[kBatch], T *(&dst)[kBatch]) {
    auto at = [&](const RopeTensor &t, int hh) { return (int64_t)b * t.batch + (int64_t)hh * t.head + (int64_t)n * t.row; };
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      if (j >= m) break;
      const int k = h >= p.heads[0], hh = h - (k ? p.heads[0] : 0);
      src[j] = static_cast<const T *>(k ? p.in[1].ptr : p.in[0].ptr) + (k ? at(p.in[1], hh) : at(p.in[0], hh));
      dst[j] = static_cast<T *>(k ? p.out[1].ptr : p.out[0].ptr) + (k ? at(p.out[1], hh) : at(p.out[0], hh));
      if (++h == HT) {
        h = 0;
        ++b;
      }
    }
  }
};

template <bool THROUGH, typename T, typename W>
__device__ __forceinline__ void rope_put(T *q, const W &v) {
  if constexpr (THROUGH) __builtin_nontemporal_store(v, reinterpret_cast<W *>(q));
  else *reinterpret_cast<W *>(q) = v;
}

// V: elements per access. INTER: interleaved pairs, a unit is one access, and with MIXED
// may hold pairs and features to copy; else a unit of pairs is an access to the first half
// and its partner in the second, and V divides the run of pairs.
template <typename T, int V, bool INTER, bool MIXED, bool THROUGH>
__global__ void __launch_bounds__(kThreads) rope_kernel(RopeArgs p) {
  constexpr int VT = V == 1 ? 2 : V;      // elements of a unit to copy (their number is even)
  typedef T vec __attribute__((ext_vector_type(V)));
  typedef T tail __attribute__((ext_vector_type(VT)));
  constexpr int NP = INTER ? V / 2 : V;   // pairs per unit
  const uint32_t idx = blockIdx.x * (uint32_t)kThreads + threadIdx.x;
  if (idx >= p.total) return;
  const uint32_t rows = fdiv(idx, p.unit_div);
  const int u = (int)(idx - rows * p.unit_div.div);
  const uint32_t grp = fdiv(rows, p.n_div);
  const int n = (int)(rows - grp * p.n_div.div);

  Slices sl(p, grp);
  const int s0 = sl.s0, s1 = sl.s1;

  // The unit's features (from e0 on, and from e1 on for the partners) and its first pair.
  const int P = p.pairs, rot = 2 * P * p.axes;
  int e0 = u * V, e1 = 0, pair = e0 / 2, axis = 0;
  bool turns = e0 < rot;
  if constexpr (!INTER) {
    const int per = P / V, nt = per * p.axes;   // units of pairs per axis, in all
    turns = u < nt;
    if (turns) {
      axis = u >= per ? 1 : 0;
      pair = (u - axis * per) * V;
      e0 = axis * 2 * P + pair;
      e1 = e0 + P;
    } else {
      e0 = rot + (u - nt) * VT;
    }
  }

  const int np = P * p.axes - pair;   // (interleaved: the pairs of the unit that are turned)
  float cs[NP], sn[NP];
  if (turns) {
    int r, c;
    sl.position(p, n, r, c);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      int pi = pair + i, ax = axis;
      if (INTER && pi >= P) {   // (a unit may cross from the row's pairs to the column's, and to features to copy)
        pi = !MIXED || i < np ? pi - P : 0;
        ax = 1;
      }
      turn_of((double)(ax ? c : r), p.freqs[pi], p, cs[i], sn[i]);
    }
  }

  // Batches of slices: all loads first, then the turns and the stores.
  for (int s = s0; s < s1; s += kBatch) {
    const T *src[kBatch];
    T *dst[kBatch];
    const int m = min(kBatch, s1 - s);
    sl.rows(p, m, n, src, dst);
    auto put = [](T *q, const auto &v) { rope_put<THROUGH>(q, v); };
    if (!INTER && !turns) {
      tail x[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j)
        if (j < m) x[j] = *reinterpret_cast<const tail *>(src[j] + e0);
#pragma unroll
      for (int j = 0; j < kBatch; ++j)
        if (j < m) put(dst[j] + e0, x[j]);
      continue;
    }
    vec a[kBatch], c[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      if (j >= m) break;
      a[j] = *reinterpret_cast<const vec *>(src[j] + e0);
      if (!INTER) c[j] = *reinterpret_cast<const vec *>(src[j] + e1);
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      if (j >= m) break;
      if (!INTER || turns) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          if constexpr (INTER) {
            const T t1 = a[j][2 * i], t2 = a[j][2 * i + 1];
            const float x1 = (float)t1, x2 = (float)t2;
            a[j][2 * i] = !MIXED || i < np ? (T)turned(x1, x2, cs[i], -sn[i]) : t1;
            a[j][2 * i + 1] = !MIXED || i < np ? (T)turned(x2, x1, cs[i], sn[i]) : t2;
          } else {
            const float x1 = (float)a[j][i], x2 = (float)c[j][i];
            a[j][i] = (T)turned(x1, x2, cs[i], -sn[i]);
            c[j][i] = (T)turned(x2, x1, cs[i], sn[i]);
          }
        }
      }
      put(dst[j] + e0, a[j]);
      if (!INTER) put(dst[j] + e1, c[j]);
    }
  }
}

// Halves by chunks: a thread owns 16 bytes of a row, whatever they hold, and finds its
// features' partners where the row's other chunks, held by the same wave, have put them
// in LDS. Features to copy stay as they are. 12 slices of 44540 rows of 64, bf16,
// 26 pairs on a grid: 34 us from memory (4.0 TB/s), 29 over one set of inputs; as units of
// one pair, 2 bytes an access, 58.
template <typename T, bool THROUGH>
__global__ void __launch_bounds__(kThreads) rope_chunks(RopeArgs p) {
  constexpr int V = 16 / (int)sizeof(T);
  typedef T vec __attribute__((ext_vector_type(V)));
  __shared__ vec lds[kBatch][kThreads];
  const int lane = threadIdx.x & 63, per = p.d / V, rows = 64 / per;   // chunks of a row, rows of a wave
  const int rr = lane / per, u = lane - rr * per;
  const uint32_t wave = blockIdx.x * (uint32_t)(kThreads / 64) + (threadIdx.x >> 6);
  const uint32_t grp = fdiv(wave, p.unit_div);
  const int n = (int)(wave - grp * p.unit_div.div) * rows + rr;
  if (grp >= p.total || rr >= rows || n >= p.N) return;
  Slices sl(p, grp);

  const int P = p.pairs, rot = 2 * P * p.axes;
  float cs[V], sn[V];
  int other[V];   // the partner's place in the wave's part of LDS, in elements
  {
    double freq[V], at[V];   // (all frequencies in flight at once)
    int r, c;
    sl.position(p, n, r, c);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int f = u * V + i, axis = f >= 2 * P ? 1 : 0, in = f - axis * 2 * P;
      const bool first = in < P, turns = f < rot;
      freq[i] = p.freqs[turns ? (first ? in : in - P) : 0];
      at[i] = (double)(axis ? c : r);
      sn[i] = first ? -1.f : 1.f;
      other[i] = lane * V + i + (turns ? (first ? P : -P) : 0);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float s;
      turn_of(at[i], freq[i], p, cs[i], s);
      sn[i] *= s;
    }
  }
  const int count = rot - u * V;   // features that are turned
  for (int s = sl.s0; s < sl.s1; s += kBatch) {
    const T *src[kBatch];
    T *dst[kBatch];
    const int m = min(kBatch, sl.s1 - s);
    sl.rows(p, m, n, src, dst);
    vec a[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j)
      if (j < m) a[j] = *reinterpret_cast<const vec *>(src[j] + u * V);
    // (a wave's LDS operations are in order, so it needs no barrier)
#pragma unroll
    for (int j = 0; j < kBatch; ++j)
      if (j < m) lds[j][threadIdx.x] = a[j];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      if (j >= m) break;
      const T *part = reinterpret_cast<const T *>(&lds[j][threadIdx.x & ~63]);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const T x = a[j][i];
        const float y = (float)part[other[i]];
        a[j][i] = i < count ? (T)turned((float)x, y, cs[i], sn[i]) : x;
      }
      rope_put<THROUGH>(dst[j] + u * V, a[j]);
    }
    asm volatile("" ::: "memory");
  }
}

// Shares `work` threads per slice out; returns how many groups of slices there are.
int64_t share_slices(RopeArgs &p, int64_t work) {
  const int64_t HT = p.heads[0] + p.heads[1], want = (int64_t)device_cu_count() * 2048;
  const int64_t most = p.pos_stride ? HT : HT * p.B;
  const int64_t run = std::max<int64_t>(1, std::min(work * HT * p.B / want, most));
  p.run = (int32_t)run;
  p.groups = (int32_t)((most + run - 1) / run);
  return (int64_t)p.groups * (p.pos_stride ? p.B : 1);
}
// A call that moves more than the caches hold.
bool goes_through(const RopeArgs &p, int es) {
  return 2 * p.B * (int64_t)(p.heads[0] + p.heads[1]) * p.N * p.d * es > (256LL << 20);
}

template <typename T, int V, bool INTER, bool MIXED>
hipError_t launch(RopeArgs &p, hipStream_t s) {
  const int rot = 2 * p.pairs * p.axes;
  const int units = INTER ? p.d / V : rot / (2 * V) + (p.d - rot) / (V == 1 ? 2 : V);
  p.unit_div = make_fastdiv((uint32_t)units);
  p.n_div = make_fastdiv((uint32_t)p.N);
  const int64_t per_slice = (int64_t)units * p.N, total = per_slice * share_slices(p, per_slice);
  p.total = (uint32_t)total;
  const dim3 grid((uint32_t)((total + kThreads - 1) / kThreads));
  if (goes_through(p, sizeof(T))) hipLaunchKernelGGL((rope_kernel<T, V, INTER, MIXED, true>), grid, dim3(kThreads), 0, s, p);
  else hipLaunchKernelGGL((rope_kernel<T, V, INTER, MIXED, false>), grid, dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

// Waves that hold the N rows of a slice (rows of up to 1 KiB).
int64_t chunk_waves(const RopeArgs &p, int es) {
  const int rows = 64 / (p.d * es / 16);
  return (p.N + rows - 1) / rows;
}

template <typename T>
hipError_t launch_chunks(RopeArgs &p, hipStream_t s) {
  const int64_t waves = chunk_waves(p, sizeof(T)), groups = share_slices(p, 64 * waves);
  p.unit_div = make_fastdiv((uint32_t)waves);
  p.total = (uint32_t)groups;
  constexpr int PER = kThreads / 64;
  const dim3 grid((uint32_t)((waves * groups + PER - 1) / PER));
  if (goes_through(p, sizeof(T))) hipLaunchKernelGGL((rope_chunks<T, true>), grid, dim3(kThreads), 0, s, p);
  else hipLaunchKernelGGL((rope_chunks<T, false>), grid, dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_any(RopeArgs &p, hipStream_t s) {
  constexpr int V = 16 / (int)sizeof(T);
  if (p.interleaved) return 2 * p.pairs * p.axes % V ? launch<T, V, true, true>(p, s) : launch<T, V, true, false>(p, s);
  // Halves: the chunks for rows that a wave holds (up to 1 KiB), but for bf16 pairs that
  // fill accesses, where both take the same time on many rows and the chunks, whose
  // threads turn every feature, longer on few (65536 rows of 10 x 64, 32 turned, fp32: 63
  // against 70 us; 320 rows of 64, bf16: 7.6 against 3.8).
  // (A batch of short rows with positions of their own may need more waves than a launch has.)
  if (p.d <= 64 * V && (V == 4 || p.pairs % V) && 64 * chunk_waves(p, sizeof(T)) * (p.pos_stride ? p.B : 1) < (1LL << 31))
    return launch_chunks<T>(p, s);
  return p.pairs % V ? launch<T, 1, false, false>(p, s) : launch<T, V, false, false>(p, s);
}

}  // namespace

hipError_t launch_rope(RopeArgs p, hla_dtype dtype, hipStream_t s) {
  return dtype == HLA_BF16 ? launch_any<__bf16>(p, s) : launch_any<float>(p, s);
}

}  // namespace hla
