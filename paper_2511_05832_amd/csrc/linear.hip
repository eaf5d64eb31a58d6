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
  // one step of 8 contracted elements (lane half h: elements KT / 2 h + 4 s .. + 3 of the stage)
  static __device__ __forceinline__ void mma(const Op &a, const Op &b, f32x16 &acc) {
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], acc, 0, 0, 0);
  }
};

// One operand's tile of R rows (or columns) by a stage of the contraction, in LDS: KB
// bytes of it per row, KB / 32 steps.
//  TR = false: R rows of KB bytes, 16-byte chunk c at c ^ (row % 8) (KB = 128) or c ^
//  (row / 2 % 4) (KB = 64), which puts the rows of a read on separate banks.
//  TR = true: the stage's elements as rows of R values, as in memory; bf16: chunk c of
//  row r at c ^ (2 (r % 4) + r / 8 % 2), which keeps the transposing reads (four rows
//  by two chunks) on separate banks; fp32 is read a value per lane, rows as they are.
template <typename T, int R, bool TR, int NT, int KB>
struct Operand {
  static constexpr int V = Type<T>::V, KT = KB / (int)sizeof(T), BYTES = R * KB;
  static constexpr int COPIES = BYTES / 16 / NT;      // per thread and stage
  static constexpr int PER = TR ? R / V : KB / 16;    // chunks per row in LDS
  static_assert(BYTES / 16 % NT == 0, "copies must split evenly");
  uint32_t off[COPIES];   // byte offset of each copy from the stage's first element
  const char *base;       // first element of the tile at contraction index 0
  int64_t step;           // bytes per stage

  static __device__ __forceinline__ int swz(int row) {
    if (!TR) return KB == 128 ? row & 7 : (row >> 1) & 3;
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
template <typename T, int R, bool TR, int NBLK, int KB>
struct Reader {
  using Op = typename Type<T>::Op;
  static constexpr int KT = KB / (int)sizeof(T);
  int at[NBLK], sw;
  __device__ __forceinline__ void init(int first, int lane) {
    const int col = lane & 31, half = lane >> 5;
    if constexpr (!TR) {
      const int x = KB == 128 ? col & 7 : (col >> 1) & 3;
      sw = ((sizeof(T) == 2 ? half : KB / 32 * half) ^ x) * 16;
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
      for (int b = 0; b < NBLK; ++b) at[b] = KT / 2 * half * R * 4 + (first + 32 * b + col) * 4;
    }
  }
  // this lane's operand of block b at step s
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

constexpr int kGroup = 8;   // tiles along NA that are walked together (4: 2% slower, 16384 x 4096 by 1024)

enum Epilogue { EPI_LAYER = 0, EPI_PLAIN = 1, EPI_PART = 2 };

struct GemmArgs {
  const void *a, *b;
  int64_t lda, ldb;          // elements between memory rows
  int32_t NA, NB, KC;        // output columns, rows; contraction
  int32_t stages;            // stages per split
  const void *bias;
  void *residual, *out, *pre;
  float *part;               // [splits, NB, NA]
  int32_t act;
  int32_t na;                // tiles along NA
  FastDiv gdiv, tdiv;        // division by the tiles of a group, and by all tiles of a split
};

template <typename T>
using Vec = T __attribute__((ext_vector_type(Type<T>::V)));
// A result's chunk past the caches (16384 x 4096 results with their z and a residual 194
// -> 182 us).
template <typename T>
__device__ __forceinline__ void store_through(T *p, const T &v) {
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<u32x4 *>(p));
}
template <typename T>
__device__ __forceinline__ void add_bias(const GemmArgs &p, int f, float (&z)[Type<T>::V]) {
  if (!p.bias) return;
  const Vec<T> b = *reinterpret_cast<const Vec<T> *>(static_cast<const T *>(p.bias) + f);
#pragma unroll
  for (int e = 0; e < Type<T>::V; ++e) z[e] += (float)b[e];
}
// The chunk at byte `off` from row `row` (the same for a wave, and its address scalar) on.
template <typename T>
__device__ __forceinline__ Vec<T> *chunk(const GemmArgs &p, void *out, int row, uint32_t off) {
  return reinterpret_cast<Vec<T> *>(static_cast<char *>(out) + (int64_t)row * p.NA * (int)sizeof(T) + off);
}
// V consecutive results of the layer from z (fp32) on.
template <typename T>
__device__ __forceinline__ void finish(const GemmArgs &p, float (&z)[Type<T>::V], const Vec<T> &residual, int row,
                                       uint32_t off) {
  constexpr int V = Type<T>::V;
  Vec<T> o;
  if (p.pre) {
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = (T)z[e];
    store_through(chunk<T>(p, p.pre, row, off), o);
  }
  apply_act<sizeof(T) == 4>(p.act, z);
  if (p.residual) {
#pragma unroll
    for (int e = 0; e < V; ++e) z[e] += (float)residual[e];
  }
#pragma unroll
  for (int e = 0; e < V; ++e) o[e] = (T)z[e];
  store_through(chunk<T>(p, p.out, row, off), o);
}

// Output tiles of TB rows by TA columns by WA x WB waves, a ring of RING stages of KB
// bytes of every row, filled by the 16-byte LDS DMA. What bounds it, in 256 x 256 tiles:
// the matrix cores and the LDS reads that feed them, about alike, then the stores, which
// one workgroup per CU does not hide. 16384 x 4096 results in bf16, over one set of inputs:
// 97 us per 1000 contracted elements (1.38 PFLOP/s) and 36 to 39 us besides; with bias and
// gelu 18 us more, and with the residual and the stored pre-activation 37 (403 MB in all).
// From memory the three take 172, 184 and 198 us, 139, 157 and 176 over one set.
template <typename T, int TA, int TB, int WA, int WB, int KB, int RING>
struct Shape {
  static constexpr int PITCH = TA + 4;   // floats of a staged output row
  static constexpr int RINGS = RING * (TA + TB) * KB, STAGED = WB * 32 * PITCH * 4;
  static constexpr int LDS = RINGS > STAGED ? RINGS : STAGED;
};

// Workgroup `block` of `blocks`.
template <typename T, int TA, int TB, int WA, int WB, int KB, int RING, bool AT, bool BT, int EPI>
__device__ __forceinline__ void gemm_tile(const GemmArgs &p, int block, int blocks, char *lds) {
  constexpr int NT = 64 * WA * WB, V = Type<T>::V, KT = KB / (int)sizeof(T);
  constexpr int AB = TA / WA / 32, BB = TB / WB / 32;
  using OA = Operand<T, TA, AT, NT, KB>;
  using OB = Operand<T, TB, BT, NT, KB>;
  constexpr int LPT = OA::COPIES + OB::COPIES;
  static_assert(LPT * (RING - 2) < 64, "vmcnt range");
  constexpr int STAGE = OA::BYTES + OB::BYTES;
  constexpr int PITCH = Shape<T, TA, TB, WA, WB, KB, RING>::PITCH;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int wa = wave % WA, wb = wave / WA;
  const int logical = xcd_remap(block, blocks);
  const int sp = (int)fdiv((uint32_t)logical, p.tdiv), tile = logical - sp * (int)p.tdiv.div;
  // Columns of kGroup tiles, row by row: the workgroups that run at once on an XCD share
  // few slices of either operand, and the group's A tiles stay in its L2.
  const int grp = (int)fdiv((uint32_t)tile, p.gdiv), in = tile - grp * (int)p.gdiv.div;
  const int wide = min(kGroup, p.na - grp * kGroup);
  const int tb = wide == kGroup ? in / kGroup : in / wide, ta = grp * kGroup + in - tb * wide;
  const int a0 = ta * TA, b0 = tb * TB;
  const int s0 = sp * p.stages, ns = min(p.stages, (p.KC + KT - 1) / KT - s0);

  OA oa;
  OB ob;
  oa.init(static_cast<const T *>(p.a), p.lda, a0, p.NA, wave, lane);
  ob.init(static_cast<const T *>(p.b), p.ldb, b0, p.NB, wave, lane);
  auto issue = [&](int i) {
    char *dst = lds + (i % RING) * STAGE;
    const int left = p.KC - (s0 + i) * KT;
    oa.issue(s0 + i, left, dst, wave, lane);
    ob.issue(s0 + i, left, dst + OA::BYTES, wave, lane);
  };
  Reader<T, TA, AT, AB, KB> ra;
  Reader<T, TB, BT, BB, KB> rb;
  ra.init(wa * 32 * AB, lane);
  rb.init(wb * 32 * BB, lane);
  // The sums start at the bias: slots 4 g .. + 3 of block x are columns 8 g + 4 half .. of it.
  f32x16 start[AB] = {};
  if constexpr (EPI == EPI_LAYER) {
    typedef T T4 __attribute__((ext_vector_type(4)));
    if (p.bias) {
#pragma unroll
      for (int i = 0; i < 4 * AB; ++i) {
        const int f = a0 + (wa * AB + i / 4) * 32 + 8 * (i % 4) + 4 * half;
        const T4 v = f < p.NA ? *reinterpret_cast<const T4 *>(static_cast<const T *>(p.bias) + f) : T4{};
#pragma unroll
        for (int e = 0; e < 4; ++e) start[i / 4][i % 4 * 4 + e] = (float)v[e];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < RING - 1; ++i)
    if (i < ns) issue(i);
  f32x16 acc[AB][BB];
#pragma unroll
  for (int x = 0; x < AB; ++x)
#pragma unroll
    for (int y = 0; y < BB; ++y) acc[x][y] = start[x];
  for (int i = 0; i < ns; ++i) {
    // stage i has landed, and every wave is done with stage i - 1
    wait_tiles_then_barrier<LPT, RING - 2>(min(RING - 2, ns - 1 - i));
    if (i + RING - 1 < ns) issue(i + RING - 1);
    const char *st = lds + (i % RING) * STAGE;
#pragma unroll
    for (int s = 0; s < KB / 32; ++s) {
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
  // (x, y) holds row 32 y + col, slots 4g .. 4g + 3 columns 8g + 4 half .. The barriers
  // wait for LDS only: the stores of one pass drain under the next, and under the next
  // workgroup's first stages.
  float *stage = reinterpret_cast<float *>(lds);
  constexpr int W = EPI == EPI_PART ? 4 : V;       // values per lane and store
  constexpr int CPR = TA / W, ROWS = WB * 32, IT = ROWS * CPR / NT;
  static_assert(ROWS * CPR % NT == 0 && NT % CPR == 0 && 32 % (NT / CPR) == 0,
                "stores must split evenly, a lane's all in one column chunk and one row of a run");
  const int c = (int)threadIdx.x % CPR, f = a0 + c * W, lr = (int)threadIdx.x / CPR;
  // Store j of pass y: row row_at(y, j) + lr, whose first part is the same for all lanes.
  auto row_at = [&](int y, int j) {
    const int r = j * (NT / CPR);
    return b0 + (r >> 5) * 32 * BB + 32 * y + (r & 31);
  };
  const uint32_t off = (uint32_t)(lr * p.NA + f) * (uint32_t)(EPI == EPI_PART ? 4 : sizeof(T));
  Vec<T> res[IT] = {};
#pragma unroll
  for (int y = 0; y < BB; ++y) {
    if constexpr (EPI == EPI_LAYER) {   // the residual's rows, in flight while the pass is staged
      if (p.residual) {
#pragma unroll
        for (int j = 0; j < IT; ++j)
          if (lr < p.NB - row_at(y, j) && f < p.NA) res[j] = *chunk<T>(p, p.residual, row_at(y, j), off);
      }
    }
    wait_then_barrier<63>();
#pragma unroll
    for (int x = 0; x < AB; ++x)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4 *>(stage + (wb * 32 + col) * PITCH + (wa * AB + x) * 32 + 8 * g + 4 * half) =
            f32x4{acc[x][y][4 * g], acc[x][y][4 * g + 1], acc[x][y][4 * g + 2], acc[x][y][4 * g + 3]};
    wait_then_barrier<63>();
#pragma unroll
    for (int j = 0; j < IT; ++j) {
      const int row = row_at(y, j);
      if (lr >= p.NB - row || f >= p.NA) continue;
      const float *src = stage + (j * (NT / CPR) + lr) * PITCH + c * W;
      if constexpr (EPI == EPI_PART) {
        char *dst = reinterpret_cast<char *>(p.part + ((int64_t)sp * p.NB + row) * p.NA);
        *reinterpret_cast<f32x4 *>(dst + off) = *reinterpret_cast<const f32x4 *>(src);
      } else {
        float z[V];
#pragma unroll
        for (int e = 0; e < V; e += 4) *reinterpret_cast<f32x4 *>(z + e) = *reinterpret_cast<const f32x4 *>(src + e);
        if constexpr (EPI == EPI_LAYER) {
          finish<T>(p, z, res[j], row, off);
        } else {
          Vec<T> o;
#pragma unroll
          for (int e = 0; e < V; ++e) o[e] = (T)z[e];
          store_through(chunk<T>(p, p.out, row, off), o);
        }
      }
    }
  }
}

template <typename T, int TA, int TB, int WA, int WB, int KB, int RING, bool AT, bool BT, int EPI>
__global__ void __launch_bounds__(64 * WA * WB, (KB == 64 ? 8 : 2)) gemm_kernel(GemmArgs p) {
  __shared__ __attribute__((aligned(16))) char lds[Shape<T, TA, TB, WA, WB, KB, RING>::LDS];
  gemm_tile<T, TA, TB, WA, WB, KB, RING, AT, BT, EPI>(p, blockIdx.x, gridDim.x, lds);
}

// dx and dW of a small layer in one launch (`first` workgroups of dx), in 64 x 64 tiles
// and possibly parts: neither fills the CUs by itself (part = null: the result itself).
template <typename T>
__global__ void __launch_bounds__(256, 2) gemm_pair_kernel(GemmArgs dx, GemmArgs dw, int first) {
  constexpr int RING = sizeof(T) == 4 ? 2 : 4;
  __shared__ __attribute__((aligned(16))) char lds[Shape<T, 64, 64, 2, 2, 128, RING>::LDS];
  const int block = blockIdx.x;
  if (block < first) {
    if (dx.part) gemm_tile<T, 64, 64, 2, 2, 128, RING, true, false, EPI_PART>(dx, block, first, lds);
    else gemm_tile<T, 64, 64, 2, 2, 128, RING, true, false, EPI_PLAIN>(dx, block, first, lds);
  } else {
    if (dw.part) gemm_tile<T, 64, 64, 2, 2, 128, RING, true, true, EPI_PART>(dw, block - first, gridDim.x - first, lds);
    else gemm_tile<T, 64, 64, 2, 2, 128, RING, true, true, EPI_PLAIN>(dw, block - first, gridDim.x - first, lds);
  }
}

// The layer for few tokens (T <= 16 NB). What bounds it: reading W once. A workgroup
// takes 16 features, its waves share the contraction in runs of 128 bytes a row; rows
// of W go from memory into operands of the 16 x 16 products (A = features, B = tokens),
// 1 KiB per load, with no stop in LDS. The waves' sums are added through LDS. 4 tokens,
// 2048 -> 8192, bf16: 10.5 us with the weights from memory (3.2 TB/s), 8.2 where the caches
// hold them; with 4 waves and the same loads in flight per wave 2.4 more, with 16 waves 1.8.
constexpr int kFewWaves = 8;
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

template <typename T, int NB>
__global__ void __launch_bounds__(64 * kFewWaves) few_kernel(GemmArgs p) {
  constexpr int NW = kFewWaves, V = Type<T>::V, RUN = 128 / (int)sizeof(T), UNROLL = NB == 1 ? 4 : 2;
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
    Vec<T> r = {};
    const uint32_t off = (uint32_t)f * (uint32_t)sizeof(T);
    if (p.residual) r = *chunk<T>(p, p.residual, t, off);
    add_bias<T>(p, f, z);
    finish<T>(p, z, r, t, off);
  }
}

// dz = dy act'(z) (when `dz` is given), and partial column sums of dz for the bias: a
// workgroup takes 32 chunks of columns by a run of rows. Where one run holds them all the
// sums are the bias' gradient itself (`db`), which saves the adding launch. Bound by HBM:
// 16384 x 4096, gelu, bf16 72 us (5.6 TB/s).
template <typename T>
__global__ void __launch_bounds__(256) dz_kernel(const T *dy, const T *pre, T *dz, float *sums, T *db, int T_,
                                                 int F, int rows, int act) {
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
        float slope[V];
#pragma unroll
        for (int e = 0; e < V; ++e) slope[e] = (float)z[e];
        apply_grad<sizeof(T) == 4>(act, slope);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = (float)g[e] * slope[e];
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
  if (!sums && !db) return;
#pragma unroll
  for (int e = 0; e < V; ++e) part[ry][cx * V + e] = s[e];
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * V; i += 256) {
    const int f = blockIdx.x * 32 * V + i;
    float t = 0.f;
#pragma unroll
    for (int y = 0; y < 8; ++y) t += part[y][i];
    if (f >= F) continue;
    if (db) db[f] = (T)t;
    else sums[(int64_t)blockIdx.y * F + f] = t;
  }
}

// out[i] = sum over n partial sums of part[s * len + i], four values per thread, for up
// to three results in one launch (a launch takes 3 to 5 us by itself). Where a short
// result has many parts, `ways` threads share them and are added through LDS, in order
// (25860 tokens, 752 -> 72, whose bias gradient has 72 values of 809 parts: the backward 72 -> 43 us).
struct SumJob {
  const float *part;
  void *out;
  int64_t len;
  int32_t n, ways, blocks;   // blocks = 0: nothing to do
};
struct SumJobs {
  SumJob job[3];
};

template <typename T>
__global__ void __launch_bounds__(256) sum_kernel(SumJobs jobs) {
  __shared__ f32x4 lds[256];
  int block = blockIdx.x, j = 0;
  while (j < 2 && block >= jobs.job[j].blocks) block -= jobs.job[j++].blocks;
  const SumJob &w = jobs.job[j];
  const int per = 256 / w.ways, way = (int)threadIdx.x / per, slot = (int)threadIdx.x - way * per;
  const int64_t i = ((int64_t)block * per + slot) * 4;
  f32x4 s = {};
  if (i < w.len) {
#pragma unroll 8
    for (int k = way; k < w.n; k += w.ways) s += *reinterpret_cast<const f32x4 *>(w.part + k * w.len + i);
  }
  if (w.ways > 1) {
    lds[threadIdx.x] = s;
    __syncthreads();
    if (way == 0)
      for (int k = 1; k < w.ways; ++k) s += lds[slot + k * per];
  }
  if (way || i >= w.len) return;
  T *out = static_cast<T *>(w.out) + i;
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<f32x4 *>(out) = s;
  } else {
    bf16x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (__bf16)s[e];
    *reinterpret_cast<bf16x4 *>(out) = o;
  }
}

SumJob sum_job(const float *part, void *out, int64_t len, int n) {
  int ways = 1;
  while (ways < 32 && n >= 16 * ways && len / 4 * ways < 256 * (int64_t)device_cu_count()) ways *= 2;
  const int per = 256 / ways;
  return {part, out, len, n, ways, (int32_t)((len / 4 + per - 1) / per)};
}

// The layer's epilogue over partial sums of its products: V columns of a row per thread.
template <typename T>
__global__ void __launch_bounds__(256) finish_kernel(GemmArgs p, int n) {
  constexpr int V = Type<T>::V;
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * V, len = (int64_t)p.NB * p.NA;
  if (i >= len) return;
  const int row = (int)(i / p.NA);
  const int f = (int)(i - (int64_t)row * p.NA);
  float z[V] = {};
#pragma unroll 4
  for (int k = 0; k < n; ++k)
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      const f32x4 x = *reinterpret_cast<const f32x4 *>(p.part + k * len + i + e);
#pragma unroll
      for (int j = 0; j < 4; ++j) z[e + j] += x[j];
    }
  Vec<T> r = {};
  const uint32_t off = (uint32_t)f * (uint32_t)sizeof(T);
  if (p.residual) r = *chunk<T>(p, p.residual, row, off);
  add_bias<T>(p, f, z);
  finish<T>(p, z, r, row, off);
}

// ---------------------------------------------------------------------------
// Which tile, and into how many parts the contraction is split.
//  fp32: 64 x 64, 128 bytes by 2 stages (32 KiB). The matrix cores are slow enough here
//    that small tiles keep them busy, and even out (4096 tokens, 1024 -> 1024: 75 us, 128 x
//    128 79; 192 -> 768: 19 against 30).
//  bf16: 256 x 256 (128 KiB, one workgroup per CU) where such tiles fill the CUs. A long
//    contraction hides a tile's first stage and its epilogue (16384 x 1024 by 4096: 112
//    us, 128 x 128 131); a short one wants the epilogue beside another workgroup's
//    products. 65536 tokens, K -> 768, with gelu / without, against 128 x 128 by stages
//    of 64 bytes: K = 192 48.7 / 35.7 against 44.9 / 39.4 us, K = 256 53.1 / 40.3 against
//    51.9 / 45.4, K = 384 63.3 / 49.0 against 66.4 / 61.7. So from 256 on, and without an
//    epilogue from 128 on. Or, where parts are allowed, a quarter of the CUs and over
//    2048 contracted elements for each part (4096 x 1024 by 16384 in four parts 125 us,
//    128 x 128 in two 128).
//    128 x 128 where those are at least three to two CUs, or, in parts, 8 stages for
//    every workgroup (768 x 192 by 65536: 32 us, 64 x 64 37): four waves and 2 stages of
//    128 bytes, two workgroups per CU; or, for a layer of a short contraction with tiles
//    for four, eight waves and 2 stages of 64 bytes, four workgroups per CU (65536 tokens,
//    192 -> 768, gelu: 44.9 us against 49.7; at two to a CU, 8192 tokens, 192 -> 1024:
//    12.1 against 11.6).
//    64 x 64 by 4 stages otherwise (2048 tokens, 1024 -> 1024: 11 us, 128 x 128 16).
// Parts: as many as fill the CUs' workgroups, of at least four stages each; fp32 gradients,
// two of which run at once: three to two CUs (4096 tokens, 192 -> 768, the whole step: 58.1
// us, with one to a CU 60.0, two 61.0, three 63.8; dx and dW one after the other 65.9).
struct Plan {
  int tile, kb;   // tile side, bytes of contraction per stage
  int splits;
  int stages;     // per split
};

template <typename T>
Plan plan_of(int64_t NA, int64_t NB, int64_t KC, bool layer, bool parts) {
  const int64_t cus = device_cu_count();
  auto tiles = [&](int t) { return ((NA + t - 1) / t) * ((NB + t - 1) / t); };
  auto make = [&](int tile, int kb, int64_t wgs, int64_t least) {
    const int64_t stages = (KC + kb / (int64_t)sizeof(T) - 1) / (kb / (int64_t)sizeof(T));
    const int64_t splits = parts ? std::max<int64_t>(1, std::min(wgs / tiles(tile), stages / least)) : 1;
    Plan p = {tile, kb, 1, (int)((stages + splits - 1) / splits)};
    p.splits = (int)((stages + p.stages - 1) / p.stages);
    return p;
  };
  if (sizeof(T) == 4) return make(64, 128, (layer ? 4 : 3) * cus / 2, 4);
  const int64_t n256 = tiles(256), n128 = tiles(128);
  const bool fills = n256 * 5 >= (n256 + cus - 1) / cus * cus * 4;   // four fifths of its rounds
  if (KC >= (layer ? 256 : 128) && fills) return make(256, 128, cus, 4);
  if (parts && !layer && 4 * n256 >= cus && KC * n256 / cus >= 2048) return make(256, 128, cus, 4);
  if (layer && KC < 256 && n128 >= 4 * cus) return make(128, 64, 1, 1);
  if (2 * n128 >= 3 * cus) return make(128, 128, 2 * cus, 4);
  if (parts && !layer && n128 * ((KC + 63) / 64) >= 16 * cus) return make(128, 128, 2 * cus, 4);
  return make(64, 128, 2 * cus, layer ? 8 : 4);
}

// Completes the arguments of a product; returns its workgroups.
uint32_t set_plan(GemmArgs &p, const Plan &plan) {
  const int64_t na = (p.NA + plan.tile - 1) / plan.tile, nb = (p.NB + plan.tile - 1) / plan.tile;
  p.stages = plan.stages;
  p.na = (int32_t)na;
  p.gdiv = make_fastdiv((uint32_t)(kGroup * nb));
  p.tdiv = make_fastdiv((uint32_t)(na * nb));
  return (uint32_t)(na * nb * plan.splits);
}

// (A layer's larger tiles are taken where they are more than half of the workgroups
// that plan_of counts on, so they are never in parts.)
template <typename T, bool AT, bool BT, int EPI>
hipError_t launch_gemm(GemmArgs &p, const Plan &plan, hipStream_t s) {
  const dim3 grid(set_plan(p, plan));
  if constexpr (sizeof(T) == 4) {
    hipLaunchKernelGGL((gemm_kernel<T, 64, 64, 2, 2, 128, 2, AT, BT, EPI>), grid, dim3(256), 0, s, p);
  } else if constexpr (EPI == EPI_PART && !AT) {
    hipLaunchKernelGGL((gemm_kernel<T, 64, 64, 2, 2, 128, 4, AT, BT, EPI>), grid, dim3(256), 0, s, p);
  } else {
    if (plan.tile == 256) {
      hipLaunchKernelGGL((gemm_kernel<T, 256, 256, 4, 2, 128, 2, AT, BT, EPI>), grid, dim3(512), 0, s, p);
    } else if (plan.tile == 64) {
      hipLaunchKernelGGL((gemm_kernel<T, 64, 64, 2, 2, 128, 4, AT, BT, EPI>), grid, dim3(256), 0, s, p);
    } else if (plan.kb == 128) {
      hipLaunchKernelGGL((gemm_kernel<T, 128, 128, 2, 2, 128, 2, AT, BT, EPI>), grid, dim3(256), 0, s, p);
    } else if constexpr (EPI == EPI_LAYER) {
      hipLaunchKernelGGL((gemm_kernel<T, 128, 128, 4, 2, 64, 2, AT, BT, EPI>), grid, dim3(512), 0, s, p);
    }
  }
  return hipGetLastError();
}

// A product whose result is rounded to T: in one launch, or in parts that `job` adds.
template <typename T, bool AT, bool BT>
hipError_t product(GemmArgs &p, const Plan &plan, SumJob *job, hipStream_t s) {
  if (plan.splits == 1) return launch_gemm<T, AT, BT, EPI_PLAIN>(p, plan, s);
  *job = sum_job(p.part, p.out, (int64_t)p.NB * p.NA, plan.splits);
  return launch_gemm<T, AT, BT, EPI_PART>(p, plan, s);
}

constexpr int kFewTokens = 64;

template <typename T>
Plan layer_plan(const LinearArgs &a) { return plan_of<T>(a.F, a.T, a.K, true, a.parts); }

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
  p.residual = const_cast<void *>(a.residual);
  p.out = a.y;
  p.pre = a.pre;
  p.act = a.act;
  if (a.T <= kFewTokens) {
    const dim3 grid((uint32_t)((a.F + 15) / 16));
    if (a.T <= 16) hipLaunchKernelGGL((few_kernel<T, 1>), grid, dim3(64 * kFewWaves), 0, s, p);
    else if (a.T <= 32) hipLaunchKernelGGL((few_kernel<T, 2>), grid, dim3(64 * kFewWaves), 0, s, p);
    else hipLaunchKernelGGL((few_kernel<T, 4>), grid, dim3(64 * kFewWaves), 0, s, p);
    return hipGetLastError();
  }
  const Plan plan = layer_plan<T>(a);
  if (plan.splits == 1) return launch_gemm<T, false, false, EPI_LAYER>(p, plan, s);
  p.part = static_cast<float *>(a.work);
  hipError_t e = launch_gemm<T, false, false, EPI_PART>(p, plan, s);
  if (e != hipSuccess) return e;
  const int64_t n = (int64_t)a.T * a.F / Type<T>::V;
  hipLaunchKernelGGL((finish_kernel<T>), dim3((uint32_t)((n + 255) / 256)), dim3(256), 0, s, p, plan.splits);
  return hipGetLastError();
}

// dx [T, K] over F, and dW [F, K] over T.
template <typename T>
Plan dx_plan(const LinearArgs &a) { return plan_of<T>(a.K, a.T, a.F, false, true); }
template <typename T>
Plan dw_plan(const LinearArgs &a) { return plan_of<T>(a.K, a.F, a.T, false, true); }

// Rows of a run of the dz launch: workgroups for every CU four times over; all of up to 128
// where no product is in parts, so that there is nothing to add (128 tokens, 800 -> 312,
// bf16, with the bias: the host issues the backward in 17 us, not 20).
template <typename T>
int dz_rows(const LinearArgs &a) {
  if (a.T <= 128 && dx_plan<T>(a).splits == 1 && dw_plan<T>(a).splits == 1) return a.T;
  const int64_t cols = (a.F / Type<T>::V + 31) / 32;
  const int64_t runs = std::max<int64_t>(1, std::min<int64_t>((a.T + 31) / 32, 4 * device_cu_count() / cols));
  return (int)((a.T + runs - 1) / runs);
}

template <typename T>
hipError_t bwd(const LinearArgs &a, hipStream_t s) {
  constexpr int V = Type<T>::V;
  const LinearWork at = linear_bwd_work(a, sizeof(T) == 2 ? HLA_BF16 : HLA_F32);
  char *work = static_cast<char *>(a.work);
  T *dz = reinterpret_cast<T *>(work + at.dz);
  float *sums = reinterpret_cast<float *>(work + at.sums);
  const bool has_act = a.act != HLA_ACT_NONE;
  SumJobs jobs = {};   // dx, dW, db
  hipError_t e;
  if (has_act || a.db) {
    const int rows = dz_rows<T>(a);
    const dim3 grid((uint32_t)((a.F / V + 31) / 32), (uint32_t)((a.T + rows - 1) / rows));
    hipLaunchKernelGGL((dz_kernel<T>), grid, dim3(256), 0, s, static_cast<const T *>(a.dy), static_cast<const T *>(a.pre),
                       has_act ? dz : nullptr, a.db && grid.y > 1 ? sums : nullptr,
                       a.db && grid.y == 1 ? static_cast<T *>(a.db) : nullptr, a.T, a.F, rows, a.act);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (a.db && grid.y > 1) jobs.job[2] = sum_job(sums, a.db, a.F, (int)grid.y);
  }
  const void *g = has_act ? static_cast<const void *>(dz) : a.dy;
  GemmArgs x = {}, w = {};
  x.a = a.w;
  x.lda = w.lda = a.K;
  x.b = w.b = g;
  x.ldb = w.ldb = a.F;
  x.NA = w.NA = a.K;
  x.NB = w.KC = a.T;
  x.KC = w.NB = a.F;
  x.out = a.dx;
  x.part = reinterpret_cast<float *>(work + at.dx);
  w.a = a.x;
  w.out = a.dw;
  w.part = reinterpret_cast<float *>(work + at.dw);
  const Plan px = dx_plan<T>(a), pw = dw_plan<T>(a);
  if (a.dx && a.dw && px.tile == 64 && pw.tile == 64) {
    if (px.splits > 1) jobs.job[0] = sum_job(x.part, x.out, (int64_t)x.NB * x.NA, px.splits);
    else x.part = nullptr;
    if (pw.splits > 1) jobs.job[1] = sum_job(w.part, w.out, (int64_t)w.NB * w.NA, pw.splits);
    else w.part = nullptr;
    const uint32_t first = set_plan(x, px), second = set_plan(w, pw);
    hipLaunchKernelGGL((gemm_pair_kernel<T>), dim3(first + second), dim3(256), 0, s, x, w, (int)first);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  } else {
    if (a.dx && (e = product<T, true, false>(x, px, &jobs.job[0], s)) != hipSuccess) return e;
    if (a.dw && (e = product<T, true, true>(w, pw, &jobs.job[1], s)) != hipSuccess) return e;
  }
  const int64_t blocks = (int64_t)jobs.job[0].blocks + jobs.job[1].blocks + jobs.job[2].blocks;
  if (!blocks) return hipSuccess;
  hipLaunchKernelGGL((sum_kernel<T>), dim3((uint32_t)blocks), dim3(256), 0, s, jobs);
  return hipGetLastError();
}

}  // namespace

namespace {

template <typename T>
LinearWork work_of(const LinearArgs &a) {
  auto up = [](int64_t n) { return (n + 255) / 256 * 256; };
  auto parts = [&](const Plan &p, int64_t len) { return p.splits == 1 ? 0 : (int64_t)p.splits * len * 4; };
  LinearWork w;
  w.dz = 0;
  w.dx = a.act != HLA_ACT_NONE ? up((int64_t)a.T * a.F * sizeof(T)) : 0;
  w.dw = w.dx + (a.dx ? up(parts(dx_plan<T>(a), (int64_t)a.T * a.K)) : 0);
  w.sums = w.dw + (a.dw ? up(parts(dw_plan<T>(a), (int64_t)a.F * a.K)) : 0);
  const int rows = dz_rows<T>(a);
  w.bytes = w.sums + (a.db ? up((int64_t)((a.T + rows - 1) / rows) * a.F * 4) : 0);
  return w;
}

template <typename T>
int64_t layer_work(const LinearArgs &a) {
  if (a.T <= kFewTokens) return 0;
  const Plan p = layer_plan<T>(a);
  return p.splits == 1 ? 0 : (int64_t)p.splits * a.T * a.F * 4;
}

}  // namespace

// Workspace of the backward: dz, the partial sums of dx, dW and db.
LinearWork linear_bwd_work(const LinearArgs &a, hla_dtype dtype) {
  return dtype == HLA_BF16 ? work_of<__bf16>(a) : work_of<float>(a);
}
// Workspace of the forward where its contraction may be split (a.parts).
int64_t linear_fwd_work(const LinearArgs &a, hla_dtype dtype) {
  return dtype == HLA_BF16 ? layer_work<__bf16>(a) : layer_work<float>(a);
}

hipError_t launch_linear(const LinearArgs &a, hla_dtype dtype, hipStream_t s) {
  return dtype == HLA_BF16 ? fwd<__bf16>(a, s) : fwd<float>(a, s);
}
hipError_t launch_linear_bwd(const LinearArgs &a, hla_dtype dtype, hipStream_t s) {
  return dtype == HLA_BF16 ? bwd<__bf16>(a, s) : bwd<float>(a, s);
}

}  // namespace hla
