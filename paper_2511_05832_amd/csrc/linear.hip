// The token-wise linear layer with its epilogue, forward and backward (hla_linear,
// hla_linear_bwd), bf16 and fp32:
//   z = x W^T + b,  y = act(z) + residual              x [T, K], W [F, K], y [T, F]
//   dz = dy act'(z),  dx = dz W,  dW = dz^T x,  db = sum_t dz_t
// Three matrix products with one kernel. Its output [NB, NA] is the sum over c of
// A(na, c) B(nb, c); an operand's memory has the contraction index along its rows
// (y: W and x; dx: dz) or across them (dx: W; dW: x and dz), and is then read from LDS
// transposed: no operand is laid out anew in memory.
#include <algorithm>

#include "act.h"
#include "attn_common.h"

namespace hla {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// What a copy reads for a chunk past the end of the contraction.
__device__ __attribute__((aligned(16))) const uint32_t kZeros[4] = {0, 0, 0, 0};

template <typename T>
struct Type;
template <>
struct Type<__bf16> {
  static constexpr int V = 8;    // elements of a 16-byte chunk
  typedef bf16x8 Op;             // a lane's operand of one step
  // one step of 16 contracted elements (lane half h: 8 h .. 8 h + 7)
  static __device__ __forceinline__ void mma(const Op &a, const Op &b, f32x16 &acc) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
  }
};
template <>
struct Type<float> {
  static constexpr int V = 4;
  typedef f32x4 Op;
  // one step of 8 contracted elements (lane half h: elements 16 h + 4 s .. + 3 of the stage)
  static __device__ __forceinline__ void mma(const Op &a, const Op &b, f32x16 &acc) {
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], acc, 0, 0, 0);
  }
};

constexpr int KB = 128;   // bytes of contraction per stage: 64 bf16 or 32 fp32 elements, four steps

// One operand's tile of R rows (or columns) by a stage of the contraction, in LDS.
//  TR = false: R rows of KB bytes, 16-byte chunk c at c ^ (row % 8).
//  TR = true: the stage's elements as rows of R values, as in memory; bf16: chunk c of
//  row r at c ^ (2 (r % 4) + r / 8 % 2), which keeps the transposing reads (four rows
//  by two chunks) on separate banks; fp32 is read a value per lane, rows as they are.
template <typename T, int R, bool TR, int NT>
struct Operand {
  static constexpr int V = Type<T>::V, KT = KB / (int)sizeof(T), BYTES = R * KB;
  static constexpr int COPIES = BYTES / 16 / NT;      // per thread and stage
  static constexpr int PER = TR ? R / V : KB / 16;    // chunks per row in LDS
  static_assert(BYTES / 16 % NT == 0, "copies must split evenly");
  uint32_t off[COPIES];   // byte offset of each copy from the stage's first element
  const char *base;       // first element of the tile at contraction index 0
  int64_t step;           // bytes per stage

  static __device__ __forceinline__ int swz(int row) {
    if (!TR) return row & 7;
    return sizeof(T) == 2 ? (2 * (row & 3)) | ((row >> 3) & 1) : 0;
  }
  // Rows (columns) from r0 on of a matrix with n of them, ld elements between memory
  // rows. What lies past the last is read from the last and not stored.
  __device__ __forceinline__ void init(const T *p, int64_t ld, int r0, int n, int wave, int lane) {
    base = reinterpret_cast<const char *>(p + (TR ? (int64_t)r0 : r0 * ld));
    step = (TR ? KT * ld : KT) * (int64_t)sizeof(T);
#pragma unroll
    for (int j = 0; j < COPIES; ++j) {
      const int q = (j * (NT / 64) + wave) * 64 + lane, row = q / PER, c = (q % PER) ^ swz(row);
      off[j] = TR ? (uint32_t)(row * ld + min(c * V, n - V - r0)) * (uint32_t)sizeof(T)
                  : (uint32_t)(min(row, n - 1 - r0) * ld + c * V) * (uint32_t)sizeof(T);
    }
  }
  // Stage i into LDS at dst; `left` contracted elements from its first on.
  __device__ __forceinline__ void issue(int i, int left, char *dst, int wave, int lane) const {
    const char *p = base + i * step;
    if (left >= KT) {
#pragma unroll
      for (int j = 0; j < COPIES; ++j) lds_dma16_at(p, off[j], lds_addr(dst + (j * (NT / 64) + wave) * 1024));
    } else {
#pragma unroll
      for (int j = 0; j < COPIES; ++j) {
        const int q = (j * (NT / 64) + wave) * 64 + lane, row = q / PER, c = (q % PER) ^ swz(row);
        const bool in = TR ? row < left : c * V < left;
        lds_dma16(in ? p + off[j] : reinterpret_cast<const char *>(kZeros), lds_addr(dst + (j * (NT / 64) + wave) * 1024));
      }
    }
  }
};

// LDS offsets of a wave's NBLK blocks of 32 rows from row `first` of a tile on.
template <typename T, int R, bool TR, int NBLK>
struct Reader {
  using Op = typename Type<T>::Op;
  int at[NBLK], sw;
  __device__ __forceinline__ void init(int first, int lane) {
    const int col = lane & 31, half = lane >> 5;
    if constexpr (!TR) {
      sw = sizeof(T) == 2 ? (half ^ (col & 7)) * 16 : ((4 * half) ^ (col & 7)) * 16;
#pragma unroll
      for (int b = 0; b < NBLK; ++b) at[b] = (first + 32 * b + col) * KB;
    } else if constexpr (sizeof(T) == 2) {
      const int g16 = lane >> 4, i16 = lane & 15, row = 8 * (g16 >> 1) + (i16 >> 2);
#pragma unroll
      for (int b = 0; b < NBLK; ++b) {
        const int cl = first + 32 * b + 16 * (g16 & 1) + 4 * (i16 & 3);
        at[b] = row * R * 2 + (((cl >> 3) ^ ((2 * (row & 3)) | ((row >> 3) & 1))) * 16) + (cl & 7) * 2;
      }
    } else {
#pragma unroll
      for (int b = 0; b < NBLK; ++b) at[b] = 16 * half * R * 4 + (first + 32 * b + col) * 4;
    }
  }
  // this lane's operand of block b at step s (0 .. 3)
  __device__ __forceinline__ Op read(const char *tile, int b, int s) const {
    if constexpr (!TR) {
      return *reinterpret_cast<const Op *>(tile + at[b] + (sw ^ (sizeof(T) == 2 ? s * 32 : s * 16)));
    } else if constexpr (sizeof(T) == 2) {
      return lds_read_tr16x2(tile + at[b] + 16 * s * R * 2, R * 2);
    } else {
      Op x;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const float *>(tile + at[b] + (4 * s + i) * R * 4);
      return x;
    }
  }
};

enum Epilogue { EPI_LAYER = 0, EPI_PLAIN = 1, EPI_PART = 2 };

struct GemmArgs {
  const void *a, *b;
  int64_t lda, ldb;          // elements between memory rows
  int32_t NA, NB, KC;        // output columns, rows; contraction
  int32_t stages;            // stages per split
  const void *bias, *residual;
  void *out, *pre;
  float *part;               // [splits, NB, NA]
  int32_t act;
  FastDiv adiv, tdiv;        // division by the tiles along NA, and by all tiles of a split
};

// V consecutive results of the layer from z before its bias (fp32) on.
template <typename T>
__device__ __forceinline__ void finish(const GemmArgs &p, float (&z)[Type<T>::V], int64_t row, int f) {
  constexpr int V = Type<T>::V;
  typedef T vec __attribute__((ext_vector_type(V)));
  const int64_t at = row * p.NA + f;
  if (p.bias) {
    const vec b = *reinterpret_cast<const vec *>(static_cast<const T *>(p.bias) + f);
#pragma unroll
    for (int e = 0; e < V; ++e) z[e] += (float)b[e];
  }
  vec o;
  if (p.pre) {
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = (T)z[e];
    *reinterpret_cast<vec *>(static_cast<T *>(p.pre) + at) = o;
  }
  if (p.act != HLA_ACT_NONE) {
#pragma unroll
    for (int e = 0; e < V; ++e) z[e] = act_of<sizeof(T) == 4>(p.act, z[e]);
  }
  if (p.residual) {
    const vec r = *reinterpret_cast<const vec *>(static_cast<const T *>(p.residual) + at);
#pragma unroll
    for (int e = 0; e < V; ++e) z[e] += (float)r[e];
  }
#pragma unroll
  for (int e = 0; e < V; ++e) o[e] = (T)z[e];
  *reinterpret_cast<vec *>(static_cast<T *>(p.out) + at) = o;
}

// Output tiles of TB rows by TA columns by WA x WB waves, a ring of two stages.
template <typename T, int TA, int TB, int WA, int WB, bool AT, bool BT, int EPI>
__global__ void __launch_bounds__(64 * WA * WB, TA * TB > 128 * 128 ? 2 : 2) gemm_kernel(GemmArgs p) {
  constexpr int NT = 64 * WA * WB, V = Type<T>::V, KT = KB / (int)sizeof(T);
  constexpr int AB = TA / WA / 32, BB = TB / WB / 32;
  using OA = Operand<T, TA, AT, NT>;
  using OB = Operand<T, TB, BT, NT>;
  constexpr int STAGE = OA::BYTES + OB::BYTES;
  constexpr int PITCH = TA + 4;                       // floats of a staged output row
  static_assert(WB * 32 * PITCH * 4 <= 2 * STAGE, "the staged rows must fit the ring");
  __shared__ __attribute__((aligned(16))) char lds[2 * STAGE];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int wa = wave % WA, wb = wave / WA;
  const int logical = xcd_remap(blockIdx.x, gridDim.x);
  const int sp = (int)fdiv((uint32_t)logical, p.tdiv), tile = logical - sp * (int)p.tdiv.div;
  const int tb = (int)fdiv((uint32_t)tile, p.adiv), ta = tile - tb * (int)p.adiv.div;
  const int a0 = ta * TA, b0 = tb * TB;
  const int s0 = sp * p.stages, ns = min(p.stages, (p.KC + KT - 1) / KT - s0);

  OA oa;
  OB ob;
  oa.init(static_cast<const T *>(p.a), p.lda, a0, p.NA, wave, lane);
  ob.init(static_cast<const T *>(p.b), p.ldb, b0, p.NB, wave, lane);
  auto issue = [&](int i) {
    char *dst = lds + (i & 1) * STAGE;
    const int left = p.KC - (s0 + i) * KT;
    oa.issue(s0 + i, left, dst, wave, lane);
    ob.issue(s0 + i, left, dst + OA::BYTES, wave, lane);
  };
  Reader<T, TA, AT, AB> ra;
  Reader<T, TB, BT, BB> rb;
  ra.init(wa * 32 * AB, lane);
  rb.init(wb * 32 * BB, lane);
  f32x16 acc[AB][BB];
#pragma unroll
  for (int x = 0; x < AB; ++x)
#pragma unroll
    for (int y = 0; y < BB; ++y) acc[x][y] = f32x16{};

  if (ns > 0) issue(0);
  for (int i = 0; i < ns; ++i) {
    wait_then_barrier<0>();   // stage i has landed, and every wave is done with stage i - 1
    if (i + 1 < ns) issue(i + 1);
    const char *st = lds + (i & 1) * STAGE;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      typename Type<T>::Op xa[AB], xb[BB];
#pragma unroll
      for (int x = 0; x < AB; ++x) xa[x] = ra.read(st, x, s);
#pragma unroll
      for (int y = 0; y < BB; ++y) xb[y] = rb.read(st + OA::BYTES, y, s);
#pragma unroll
      for (int x = 0; x < AB; ++x)
#pragma unroll
        for (int y = 0; y < BB; ++y) Type<T>::mma(xa[x], xb[y], acc[x][y]);
    }
  }

  // Through LDS as fp32 rows, WB * 32 output rows at a time, so that the layer's
  // epilogue rounds once and memory is met in whole rows. Lane (col, half) of block
  // (x, y) holds row 32 y + col, slots 4g .. 4g + 3 columns 8g + 4 half ..
  float *stage = reinterpret_cast<float *>(lds);
#pragma unroll
  for (int y = 0; y < BB; ++y) {
    wait_then_barrier<0>();
#pragma unroll
    for (int x = 0; x < AB; ++x)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4 *>(stage + (wb * 32 + col) * PITCH + (wa * AB + x) * 32 + 8 * g + 4 * half) =
            f32x4{acc[x][y][4 * g], acc[x][y][4 * g + 1], acc[x][y][4 * g + 2], acc[x][y][4 * g + 3]};
    wait_then_barrier<0>();
    constexpr int W = EPI == EPI_PART ? 4 : V;       // values per lane and store
    constexpr int CPR = TA / W, ROWS = WB * 32;
    static_assert(ROWS * CPR % NT == 0, "stores must split evenly");
#pragma unroll 2
    for (int j = 0; j < ROWS * CPR / NT; ++j) {
      const int q = j * NT + (int)threadIdx.x, r = q / CPR, c = q % CPR;
      const int row = b0 + (r >> 5) * 32 * BB + 32 * y + (r & 31), f = a0 + c * W;
      if (row >= p.NB || f >= p.NA) continue;
      const float *src = stage + r * PITCH + c * W;
      if constexpr (EPI == EPI_PART) {
        *reinterpret_cast<f32x4 *>(p.part + ((int64_t)sp * p.NB + row) * p.NA + f) = *reinterpret_cast<const f32x4 *>(src);
      } else {
        float z[V];
#pragma unroll
        for (int e = 0; e < V; e += 4) *reinterpret_cast<f32x4 *>(z + e) = *reinterpret_cast<const f32x4 *>(src + e);
        if constexpr (EPI == EPI_LAYER) {
          finish<T>(p, z, row, f);
        } else {
          typedef T vec __attribute__((ext_vector_type(V)));
          vec o;
#pragma unroll
          for (int e = 0; e < V; ++e) o[e] = (T)z[e];
          *reinterpret_cast<vec *>(static_cast<T *>(p.out) + (int64_t)row * p.NA + f) = o;
        }
      }
    }
  }
}

// The layer for few tokens (T <= 16 NB). What bounds it: reading W once. A workgroup
// takes 16 features, its NW waves share the contraction in runs of 128 bytes a row;
// rows of W go from memory into operands of the 16 x 16 products (A = features, B =
// tokens), 1 KiB per load, with no stop in LDS. The waves' sums are added through LDS.
template <typename T>
struct Few;
template <>
struct Few<__bf16> {
  static __device__ __forceinline__ void mma(const bf16x8 &a, const bf16x8 &b, f32x4 &acc) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0);
  }
};
template <>
struct Few<float> {
  static __device__ __forceinline__ void mma(const f32x4 &a, const f32x4 &b, f32x4 &acc) {
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], acc, 0, 0, 0);
  }
};

template <typename T, int NB, int NW>
__global__ void __launch_bounds__(64 * NW) few_kernel(GemmArgs p) {
  constexpr int V = Type<T>::V, RUN = KB / (int)sizeof(T), UNROLL = NB == 1 ? 4 : 2;
  typedef typename Type<T>::Op Op;
  __shared__ __attribute__((aligned(16))) f32x4 sums[NW][NB][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g4 = lane >> 4;
  const int f0 = blockIdx.x * 16;
  // (features and tokens past the last read it and are not stored)
  const T *w = static_cast<const T *>(p.a) + (int64_t)min(f0 + l16, p.NA - 1) * p.lda + g4 * V;
  const T *x[NB];
  f32x4 acc[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    x[n] = static_cast<const T *>(p.b) + (int64_t)min(16 * n + l16, p.NB - 1) * p.ldb + g4 * V;
    acc[n] = f32x4{};
  }
  const int whole = p.KC / RUN;   // whole runs; two products of 4 V elements each
  int u = wave;
  for (; u + (UNROLL - 1) * NW < whole; u += UNROLL * NW) {
    Op a[UNROLL][2], b[UNROLL][2][NB];
#pragma unroll
    for (int i = 0; i < UNROLL; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = (u + i * NW) * RUN + h * (RUN / 2);
        a[i][h] = *reinterpret_cast<const Op *>(w + k);
#pragma unroll
        for (int n = 0; n < NB; ++n) b[i][h][n] = *reinterpret_cast<const Op *>(x[n] + k);
      }
#pragma unroll
    for (int i = 0; i < UNROLL; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int n = 0; n < NB; ++n) Few<T>::mma(a[i][h], b[i][h][n], acc[n]);
  }
  for (; u * RUN < p.KC; u += NW) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = u * RUN + h * (RUN / 2);
      const bool in = k + g4 * V < p.KC;   // (KC is a multiple of V)
      const Op a = in ? *reinterpret_cast<const Op *>(w + k) : Op{};
#pragma unroll
      for (int n = 0; n < NB; ++n) Few<T>::mma(a, in ? *reinterpret_cast<const Op *>(x[n] + k) : Op{}, acc[n]);
    }
  }
#pragma unroll
  for (int n = 0; n < NB; ++n) sums[wave][n][lane] = acc[n];
  __syncthreads();
  // lane (l16, g4): token l16 of block n, features 4 g4 .. + 3; V consecutive features
  // of a token per thread
  constexpr int PER = 16 / V;
  for (int i = threadIdx.x; i < 16 * NB * PER; i += 64 * NW) {
    const int c = i % PER, t = i / PER, f = f0 + c * V;
    if (t >= p.NB || f >= p.NA) continue;
    float z[V];
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      f32x4 s = {};
      for (int v = 0; v < NW; ++v) s += sums[v][t / 16][(c * V + e) / 4 * 16 + t % 16];
#pragma unroll
      for (int j = 0; j < 4; ++j) z[e + j] = s[j];
    }
    finish<T>(p, z, t, f);
  }
}

// dz = dy act'(z) (when `dz` is given), and partial column sums of dz for the bias: a
// workgroup takes 32 chunks of columns by a run of rows.
template <typename T>
__global__ void __launch_bounds__(256) dz_kernel(const T *dy, const T *pre, T *dz, float *sums, int T_, int F,
                                                 int rows, int act) {
  constexpr int V = Type<T>::V;
  typedef T vec __attribute__((ext_vector_type(V)));
  __shared__ float part[8][32 * V];
  const int cx = threadIdx.x & 31, ry = threadIdx.x >> 5;
  const int c = (blockIdx.x * 32 + cx) * V;
  const int r1 = min((int)(blockIdx.y + 1) * rows, T_);
  float s[V] = {};
  if (c < F) {
#pragma unroll 4
    for (int r = blockIdx.y * rows + ry; r < r1; r += 8) {
      const int64_t at = (int64_t)r * F + c;
      vec g = *reinterpret_cast<const vec *>(dy + at);
      if (dz) {
        const vec z = *reinterpret_cast<const vec *>(pre + at);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = (float)g[e] * act_grad<sizeof(T) == 4>(act, (float)z[e]);
          s[e] += d;
          g[e] = (T)d;
        }
        *reinterpret_cast<vec *>(dz + at) = g;
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) s[e] += (float)g[e];
      }
    }
  }
  if (!sums) return;
#pragma unroll
  for (int e = 0; e < V; ++e) part[ry][cx * V + e] = s[e];
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * V; i += 256) {
    const int f = blockIdx.x * 32 * V + i;
    float t = 0.f;
#pragma unroll
    for (int y = 0; y < 8; ++y) t += part[y][i];
    if (f < F) sums[(int64_t)blockIdx.y * F + f] = t;
  }
}

// out[i] = sum over n partial sums of part[s * len + i], four values per thread.
template <typename T>
__global__ void __launch_bounds__(256) sum_kernel(const float *part, T *out, int64_t len, int n) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= len) return;
  f32x4 s = {};
#pragma unroll 4
  for (int k = 0; k < n; ++k) s += *reinterpret_cast<const f32x4 *>(part + k * len + i);
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<f32x4 *>(out + i) = s;
  } else {
    bf16x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (__bf16)s[e];
    *reinterpret_cast<bf16x4 *>(out + i) = o;
  }
}

// ---------------------------------------------------------------------------
// Which tile, and into how many parts the contraction is split.
struct Plan {
  int tile;       // 256, 128 or 64 a side
  int splits;
  int stages;     // per split
};

Plan plan_of(int64_t NA, int64_t NB, int64_t KC, int kt, bool splittable) {
  const int64_t cus = device_cu_count();
  auto tiles = [&](int t) { return ((NA + t - 1) / t) * ((NB + t - 1) / t); };
  Plan p;
  p.tile = tiles(256) >= cus / 2 && kt == 64 ? 256 : (tiles(128) >= cus / 2 || splittable ? 128 : 64);
  const int64_t stages = (KC + kt - 1) / kt;
  int64_t splits = 1;
  if (splittable) splits = std::max<int64_t>(1, std::min(cus / tiles(p.tile), stages / 4));
  p.stages = (int)((stages + splits - 1) / splits);
  p.splits = (int)((stages + p.stages - 1) / p.stages);
  return p;
}

template <typename T, bool AT, bool BT, int EPI>
hipError_t launch_gemm(GemmArgs &p, const Plan &plan, hipStream_t s) {
  const int64_t na = (p.NA + plan.tile - 1) / plan.tile, nb = (p.NB + plan.tile - 1) / plan.tile;
  p.stages = plan.stages;
  p.adiv = make_fastdiv((uint32_t)na);
  p.tdiv = make_fastdiv((uint32_t)(na * nb));
  const dim3 grid((uint32_t)(na * nb * plan.splits));
  if constexpr (sizeof(T) == 2) {
    if (plan.tile == 256) {
      hipLaunchKernelGGL((gemm_kernel<T, 256, 256, 4, 2, AT, BT, EPI>), grid, dim3(512), 0, s, p);
      return hipGetLastError();
    }
  }
  if (plan.tile == 128) hipLaunchKernelGGL((gemm_kernel<T, 128, 128, 2, 2, AT, BT, EPI>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((gemm_kernel<T, 64, 64, 2, 2, AT, BT, EPI>), grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

// A product whose result is rounded to T: in one launch, or in parts and their sum.
template <typename T, bool AT, bool BT>
hipError_t product(GemmArgs &p, const Plan &plan, hipStream_t s) {
  if (plan.splits == 1) return launch_gemm<T, AT, BT, EPI_PLAIN>(p, plan, s);
  hipError_t e = launch_gemm<T, AT, BT, EPI_PART>(p, plan, s);
  if (e != hipSuccess) return e;
  const int64_t len = (int64_t)p.NB * p.NA;
  hipLaunchKernelGGL((sum_kernel<T>), dim3((uint32_t)((len / 4 + 255) / 256)), dim3(256), 0, s, p.part,
                     static_cast<T *>(p.out), len, plan.splits);
  return hipGetLastError();
}

template <typename T>
hipError_t fwd(const LinearArgs &a, hipStream_t s) {
  GemmArgs p = {};
  p.a = a.w;
  p.b = a.x;
  p.lda = p.ldb = a.K;
  p.NA = a.F;
  p.NB = a.T;
  p.KC = a.K;
  p.bias = a.bias;
  p.residual = a.residual;
  p.out = a.y;
  p.pre = a.pre;
  p.act = a.act;
  if (a.T <= 64) {
    const dim3 grid((uint32_t)((a.F + 15) / 16));
    // (more waves to a workgroup where there are few workgroups)
    const bool wide = (int)grid.x >= device_cu_count();
    if (a.T <= 16) {
      if (wide) hipLaunchKernelGGL((few_kernel<T, 1, 4>), grid, dim3(256), 0, s, p);
      else hipLaunchKernelGGL((few_kernel<T, 1, 16>), grid, dim3(1024), 0, s, p);
    } else {
      if (wide) hipLaunchKernelGGL((few_kernel<T, 4, 4>), grid, dim3(256), 0, s, p);
      else hipLaunchKernelGGL((few_kernel<T, 4, 8>), grid, dim3(512), 0, s, p);
    }
    return hipGetLastError();
  }
  return launch_gemm<T, false, false, EPI_LAYER>(p, plan_of(a.F, a.T, a.K, KB / (int)sizeof(T), false), s);
}

// Runs of rows of the dz launch: workgroups for every CU four times over.
int dz_rows(const LinearArgs &a, int V) {
  const int64_t cols = (a.F / V + 31) / 32;
  const int64_t runs = std::max<int64_t>(1, std::min<int64_t>((a.T + 31) / 32, 4 * device_cu_count() / cols));
  return (int)((a.T + runs - 1) / runs);
}

template <typename T>
hipError_t bwd(const LinearArgs &a, hipStream_t s) {
  constexpr int V = Type<T>::V, KT = KB / (int)sizeof(T);
  const LinearWork w = linear_work(a, (int)sizeof(T));
  char *work = static_cast<char *>(a.work);
  T *dz = reinterpret_cast<T *>(work + w.dz);
  float *part = reinterpret_cast<float *>(work + w.part), *sums = reinterpret_cast<float *>(work + w.sums);
  const bool has_act = a.act != HLA_ACT_NONE;
  hipError_t e;
  if (has_act || a.db) {
    const int rows = dz_rows(a, V);
    const dim3 grid((uint32_t)((a.F / V + 31) / 32), (uint32_t)((a.T + rows - 1) / rows));
    hipLaunchKernelGGL((dz_kernel<T>), grid, dim3(256), 0, s, static_cast<const T *>(a.dy), static_cast<const T *>(a.pre),
                       has_act ? dz : nullptr, a.db ? sums : nullptr, a.T, a.F, rows, a.act);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (a.db) {
      hipLaunchKernelGGL((sum_kernel<T>), dim3((uint32_t)((a.F / 4 + 255) / 256)), dim3(256), 0, s, sums,
                         static_cast<T *>(a.db), (int64_t)a.F, (int)grid.y);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  const void *g = has_act ? static_cast<const void *>(dz) : a.dy;
  if (a.dx) {
    GemmArgs p = {};
    p.a = a.w;
    p.lda = a.K;
    p.b = g;
    p.ldb = a.F;
    p.NA = a.K;
    p.NB = a.T;
    p.KC = a.F;
    p.out = a.dx;
    p.part = part;
    if ((e = product<T, true, false>(p, plan_of(a.K, a.T, a.F, KT, true), s)) != hipSuccess) return e;
  }
  if (a.dw) {
    GemmArgs p = {};
    p.a = a.x;
    p.lda = a.K;
    p.b = g;
    p.ldb = a.F;
    p.NA = a.K;
    p.NB = a.F;
    p.KC = a.T;
    p.out = a.dw;
    p.part = part;
    if ((e = product<T, true, true>(p, plan_of(a.K, a.F, a.T, KT, true), s)) != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

// Workspace of the backward: dz, the products' partial sums (dx's and dW's in turn),
// the bias' partial sums.
LinearWork linear_work(const LinearArgs &a, int es) {
  const int V = 16 / es, kt = KB / es;
  auto up = [](int64_t n) { return (n + 255) / 256 * 256; };
  auto parts = [&](const Plan &p, int64_t len) { return p.splits == 1 ? 0 : (int64_t)p.splits * len * 4; };
  LinearWork w;
  w.dz = 0;
  w.part = a.act != HLA_ACT_NONE ? up((int64_t)a.T * a.F * es) : 0;
  const int64_t dx = a.dx ? parts(plan_of(a.K, a.T, a.F, kt, true), (int64_t)a.T * a.K) : 0;
  const int64_t dw = a.dw ? parts(plan_of(a.K, a.F, a.T, kt, true), (int64_t)a.F * a.K) : 0;
  w.sums = w.part + up(std::max(dx, dw));
  const int rows = dz_rows(a, V);
  w.bytes = w.sums + (a.db ? up((int64_t)((a.T + rows - 1) / rows) * a.F * 4) : 0);
  return w;
}

hipError_t launch_linear(const LinearArgs &a, hla_dtype dtype, hipStream_t s) {
  return dtype == HLA_BF16 ? fwd<__bf16>(a, s) : fwd<float>(a, s);
}
hipError_t launch_linear_bwd(const LinearArgs &a, hla_dtype dtype, hipStream_t s) {
  return dtype == HLA_BF16 ? bwd<__bf16>(a, s) : bwd<float>(a, s);
}

}  // namespace hla
