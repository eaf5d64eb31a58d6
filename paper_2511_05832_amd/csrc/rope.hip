// Rotary positions (hla_rope): every pair (x1, x2) of a row's first `rot` features is
// turned by the angle a = position * frequency,
//   y1 = m (x1 cos a - x2 sin a),   y2 = m (x2 cos a + x1 sin a),
// with -a in place of a for the way back of a gradient; the other features are copied.
//
// Bound by HBM: each row is read and written once. A thread owns one unit of a row -
// the 16-byte chunks that hold a run of pairs, or one chunk to copy - at one position,
// computes the unit's sines and cosines once, and goes through a run of (batch, head)
// slices with them, so the trigonometry (about 60 operations per pair) is shared. The
// runs are as long as leaves the chip enough threads.
//
// The angle is formed in float64 and reduced to a fraction of a turn before it is
// rounded: at position 10^5 and frequency 1 the float32 product is already 4e-3 off,
// while this is below 2e-7 up to 2^28.
#include "attn_common.h"

namespace hla {
namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;   // slices whose loads are in flight together

template <typename T>
struct Chunk {
  static constexpr int V = 16 / (int)sizeof(T);
  typedef T type __attribute__((ext_vector_type(V)));
};

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

// KIND 0: interleaved pairs, a unit is one chunk. KIND 1: halves whose length is a
// multiple of a chunk, a unit is a chunk of the first half and its partner. KIND 2: any
// other, a unit is one pair (or two features to copy), element by element.
template <typename T, int KIND>
__global__ void __launch_bounds__(kThreads) rope_kernel(RopeArgs p) {
  constexpr int V = Chunk<T>::V;
  typedef typename Chunk<T>::type vec;
  constexpr int NP = KIND == 0 ? V / 2 : (KIND == 1 ? V : 1);   // pairs per unit
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

  // The unit's features (e0, and e1 for its partner) and its first pair.
  const int P = p.pairs, rot = 2 * P * p.axes;
  int e0, e1 = 0, pair, axis;
  bool turned;
  if constexpr (KIND == 0) {
    e0 = u * V;
    turned = e0 < rot;
    pair = e0 / 2;
    axis = 0;   // (per pair below: a chunk may cross from rows to columns)
  } else {
    const int per = KIND == 1 ? P / V : P;             // units per axis
    const int nt = per * p.axes;
    turned = u < nt;
    axis = turned && u >= per ? 1 : 0;
    pair = (u - axis * per) * (KIND == 1 ? V : 1);
    if (turned) {
      e0 = KIND == 2 && p.interleaved ? 2 * (axis * P + pair) : axis * 2 * P + pair;
      e1 = KIND == 2 && p.interleaved ? e0 + 1 : e0 + P;
    } else {
      e0 = rot + (u - nt) * (KIND == 1 ? V : 2);
      e1 = e0 + 1;
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
      if (KIND == 0 && pi >= P) {
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
    if constexpr (KIND == 2) {
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (j >= m) break;
        const T t0 = src[j][e0], t1 = src[j][e1];
        const float x1 = (float)t0, x2 = (float)t1;
        dst[j][e0] = turned ? (T)(x1 * cs[0] - x2 * sn[0]) : t0;
        dst[j][e1] = turned ? (T)(x2 * cs[0] + x1 * sn[0]) : t1;
      }
    } else {
      vec a[kBatch], c[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (j >= m) break;
        a[j] = *reinterpret_cast<const vec *>(src[j] + e0);
        if (KIND == 1 && turned) c[j] = *reinterpret_cast<const vec *>(src[j] + e1);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (j >= m) break;
        if (turned) {
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            if constexpr (KIND == 0) {
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
        *reinterpret_cast<vec *>(dst[j] + e0) = a[j];
        if (KIND == 1 && turned) *reinterpret_cast<vec *>(dst[j] + e1) = c[j];
      }
    }
  }
}

template <typename T>
hipError_t launch(RopeArgs &p, hipStream_t s) {
  constexpr int V = Chunk<T>::V;
  const int rot = 2 * p.pairs * p.axes;
  int kind, units;
  if (p.interleaved && rot % V == 0) {
    kind = 0;
    units = p.d / V;
  } else if (!p.interleaved && p.pairs % V == 0) {
    kind = 1;
    units = rot / (2 * V) + (p.d - rot) / V;
  } else {
    kind = 2;
    units = p.d / 2;
  }
  p.unit_div = make_fastdiv((uint32_t)units);
  p.n_div = make_fastdiv((uint32_t)p.N);
  // Runs of slices as long as leaves every CU eight waves of threads.
  const int64_t per_slice = (int64_t)units * p.N, HT = p.heads[0] + p.heads[1];
  const int64_t want = (int64_t)device_cu_count() * 512;
  int64_t run = per_slice * HT * p.B / want;
  const int64_t most = p.pos_stride ? HT : HT * p.B;
  run = run < 1 ? 1 : (run > most ? most : run);
  p.run = (int32_t)run;
  p.groups = (int32_t)((most + run - 1) / run);
  const int64_t total = per_slice * p.groups * (p.pos_stride ? p.B : 1);
  p.total = (uint32_t)total;
  const dim3 grid((uint32_t)((total + kThreads - 1) / kThreads));
  if (kind == 0) hipLaunchKernelGGL((rope_kernel<T, 0>), grid, dim3(kThreads), 0, s, p);
  else if (kind == 1) hipLaunchKernelGGL((rope_kernel<T, 1>), grid, dim3(kThreads), 0, s, p);
  else hipLaunchKernelGGL((rope_kernel<T, 2>), grid, dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(RopeArgs p, hla_dtype dtype, hipStream_t s) {
  return dtype == HLA_BF16 ? launch<__bf16>(p, s) : launch<float>(p, s);
}

}  // namespace hla
