// Rotary positions (hla_rope): every pair (x1, x2) of a row's first `rot` features is
// turned by the angle a = position * frequency,
//   y1 = m (x1 cos a - x2 sin a),   y2 = m (x2 cos a + x1 sin a),
// with -a in place of a for the way back of a gradient; the other features are copied.
//
// Bound by HBM: each row is read and written once. A thread owns one unit of a row -
// a run of pairs that 16 bytes hold, or as many to copy - at one position, computes the
// unit's sines and cosines once, and goes through a run of (batch, head) slices with
// them, so the trigonometry (about 60 operations per pair) is shared. The runs leave the
// chip 32 waves per CU, two slices' loads in flight each. Measured: 64x64 layer, 6 heads
// of 32, batch 16, bf16 18 us (5.6 TB/s); 65536 tokens, 8 + 2 heads of 64, fp32 57 us
// (5.9 TB/s; a copy of 1 GiB 5.1).
// Results go past the caches where a call moves more than they hold (256 MB): there
// 77 -> 57 us, while at 84 MB 16.4 -> 18.4 and the next kernel finds its inputs in memory.
//
// The angle is formed in float64 and reduced to a fraction of a turn before it is
// rounded: at position 10^5 and frequency 1 the float32 product is already 4e-3 off,
// while this is below 2e-7 up to 2^28.
#include <type_traits>

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

// V: elements per access, the most that divide the run of pairs and fit 16 bytes (a
// run of an odd number of pairs in halves: 1). INTER: interleaved pairs, a unit is one
// access; else a unit of pairs is an access to the first half and its partner in the
// second.
template <typename T, int V, bool INTER, bool THROUGH>
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

  // The slices [s0, s1) of this thread: slice s is head s % HT of batch element s / HT
  // (q's heads first, then k's). Per-batch positions: a group lies in one batch element.
  const int HT = p.heads[0] + p.heads[1];
  int s0, s1, b;
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
  int h = s0 - b * HT;

  // The unit's features (from e0 on, and from e1 on for the partners) and its first pair.
  const int P = p.pairs, rot = 2 * P * p.axes;
  int e0 = u * V, e1 = 0, pair = e0 / 2, axis = 0;
  bool turned = e0 < rot;
  if constexpr (!INTER) {
    const int per = P / V, nt = per * p.axes;   // units of pairs per axis, in all
    turned = u < nt;
    if (turned) {
      axis = u >= per ? 1 : 0;
      pair = (u - axis * per) * V;
      e0 = axis * 2 * P + pair;
      e1 = e0 + P;
    } else {
      e0 = rot + (u - nt) * VT;
    }
  }

  float cs[NP], sn[NP];
  if (turned) {
    const int pos = p.pos ? p.pos[(int64_t)(p.pos_stride ? b : 0) * p.pos_stride + n] : n;
    int r = pos, c = 0;
    if (p.axes == 2) {
      r = (int)((uint32_t)pos / (uint32_t)p.grid_w);
      c = pos - r * p.grid_w;
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      int pi = pair + i, ax = axis;
      if (INTER && pi >= P) {   // (a unit may cross from the row's pairs to the column's)
        pi -= P;
        ax = 1;
      }
      turn_of((double)(ax ? c : r), p.freqs[pi], p, cs[i], sn[i]);
    }
  }

  auto at = [&](const RopeTensor &t, int hh, int bb) { return (int64_t)bb * t.batch + (int64_t)hh * t.head + (int64_t)n * t.row; };
  // Batches of slices: all loads first, then the turns and the stores.
  for (int s = s0; s < s1; s += kBatch) {
    const T *src[kBatch];
    T *dst[kBatch];
    const int m = min(kBatch, s1 - s);
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      if (j >= m) break;
      const int k = h >= p.heads[0];
      const int hh = h - (k ? p.heads[0] : 0);
      src[j] = static_cast<const T *>(k ? p.in[1].ptr : p.in[0].ptr) + (k ? at(p.in[1], hh, b) : at(p.in[0], hh, b));
      dst[j] = static_cast<T *>(k ? p.out[1].ptr : p.out[0].ptr) + (k ? at(p.out[1], hh, b) : at(p.out[0], hh, b));
      if (++h == HT) {
        h = 0;
        ++b;
      }
    }
    auto put = [](T *q, const auto &v) {
      using W = std::remove_const_t<std::remove_reference_t<decltype(v)>>;
      if constexpr (THROUGH) __builtin_nontemporal_store(v, reinterpret_cast<W *>(q));
      else *reinterpret_cast<W *>(q) = v;
    };
    if (!INTER && !turned) {
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
      if (!INTER || turned) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          if constexpr (INTER) {
            const float x1 = (float)a[j][2 * i], x2 = (float)a[j][2 * i + 1];
            a[j][2 * i] = (T)(x1 * cs[i] - x2 * sn[i]);
            a[j][2 * i + 1] = (T)(x2 * cs[i] + x1 * sn[i]);
          } else {
            const float x1 = (float)a[j][i], x2 = (float)c[j][i];
            a[j][i] = (T)(x1 * cs[i] - x2 * sn[i]);
            c[j][i] = (T)(x2 * cs[i] + x1 * sn[i]);
          }
        }
      }
      put(dst[j] + e0, a[j]);
      if (!INTER) put(dst[j] + e1, c[j]);
    }
  }
}

template <typename T, int V, bool INTER>
hipError_t launch(RopeArgs &p, hipStream_t s) {
  const int rot = 2 * p.pairs * p.axes;
  const int units = INTER ? p.d / V : rot / (2 * V) + (p.d - rot) / (V == 1 ? 2 : V);
  p.unit_div = make_fastdiv((uint32_t)units);
  p.n_div = make_fastdiv((uint32_t)p.N);
  const int64_t per_slice = (int64_t)units * p.N, HT = p.heads[0] + p.heads[1];
  const int64_t want = (int64_t)device_cu_count() * 2048;
  int64_t run = per_slice * HT * p.B / want;
  const int64_t most = p.pos_stride ? HT : HT * p.B;
  run = run < 1 ? 1 : (run > most ? most : run);
  p.run = (int32_t)run;
  p.groups = (int32_t)((most + run - 1) / run);
  const int64_t total = per_slice * p.groups * (p.pos_stride ? p.B : 1);
  p.total = (uint32_t)total;
  const dim3 grid((uint32_t)((total + kThreads - 1) / kThreads));
  const int64_t bytes = 2 * p.B * HT * p.N * p.d * (int64_t)sizeof(T);
  if (bytes > (256LL << 20)) hipLaunchKernelGGL((rope_kernel<T, V, INTER, true>), grid, dim3(kThreads), 0, s, p);
  else hipLaunchKernelGGL((rope_kernel<T, V, INTER, false>), grid, dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

// The widest access that divides the features of an axis' pairs (interleaved) or the
// pairs themselves.
template <typename T>
hipError_t launch_any(RopeArgs &p, hipStream_t s) {
  constexpr int V = 16 / (int)sizeof(T);
  if (p.interleaved) {
    const int n = 2 * p.pairs * p.axes;
    if (n % V == 0) return launch<T, V, true>(p, s);
    if (V == 8 && n % 4 == 0) return launch<T, 4, true>(p, s);
    return launch<T, 2, true>(p, s);
  }
  if (p.pairs % V == 0) return launch<T, V, false>(p, s);
  if (V == 8 && p.pairs % 4 == 0) return launch<T, 4, false>(p, s);
  if (p.pairs % 2 == 0) return launch<T, 2, false>(p, s);
  return launch<T, 1, false>(p, s);
}

}  // namespace

hipError_t launch_rope(RopeArgs p, hla_dtype dtype, hipStream_t s) {
  return dtype == HLA_BF16 ? launch_any<__bf16>(p, s) : launch_any<float>(p, s);
}

}  // namespace hla
