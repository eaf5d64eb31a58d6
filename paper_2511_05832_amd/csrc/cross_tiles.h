// The matrix products of the cross-attention kernels on 32-row blocks of a row tile in
// LDS, for bf16 (v_mfma_f32_32x32x16_bf16) and fp32 (v_mfma_f32_32x32x2_f32) behind
// one interface, so that each kernel is written once.
//
// A tile holds rows of D elements, 16-byte chunk c of row r at chunk c ^ swz(r), which
// keeps both ways of reading free of bank conflicts. A lane (col = l % 32, half =
// l / 32) stands for one row of the other operand, whose half `half` of D it holds in
// registers (Frag). Accumulators are f32x16: slot v of lane half h is row
// 16 (v/8) + 8 h + v%8 of the block (rows_times) - the rows are fed permuted, so that
// weights come out as the operand of the product that contracts over them - or column
// slots of D as columns() lists them (cols_times).
#pragma once

#include "attn_common.h"

namespace hla {

template <typename T, int D>
struct Tile;

template <int D>
struct Tile<__bf16, D> {
  static constexpr int ROW = D * 2, CPR = D / 8, NDB = D / 32, NCH = D / 16;
  typedef bf16x8 Frag[NCH];
  int row[NCH];   // by rows: chunk c of this lane's row
  int tr[NDB];    // transposed: first read of a 16-row step

  static __device__ __forceinline__ int swz(int r) {
    return D == 64 ? (2 * (r & 3)) | ((r >> 3) & 1) : (2 * ((r >> 1) & 1)) | ((r >> 3) & 1);
  }
  __device__ __forceinline__ void init(int lane) {
    const int r = row_perm(lane & 31), half = lane >> 5;
#pragma unroll
    for (int c = 0; c < NCH; ++c) row[c] = r * ROW + (((half * NCH + c) ^ swz(r)) * 16);
    // lane i of 16-lane group g reads row 8 (g/2) + i/4 (+4 in the second read) and
    // columns 32 db + 16 (g%2) + 4 (i%4); rows 4 apart have the same swizzle
    const int g16 = lane >> 4, i16 = lane & 15, tr_row = 8 * (g16 >> 1) + (i16 >> 2);
#pragma unroll
    for (int db = 0; db < NDB; ++db) {
      const int cl = db * 32 + 16 * (g16 & 1) + 4 * (i16 & 3);
      tr[db] = tr_row * ROW + (((cl >> 3) ^ swz(tr_row)) * 16) + (cl & 7) * 2;
    }
  }
  static __device__ __forceinline__ void load(Frag &f, const __bf16 *p, int half) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) f[c] = *reinterpret_cast<const bf16x8 *>(p + half * (D / 2) + 8 * c);
  }
  // <a, b> over this lane's half of D
  static __device__ __forceinline__ float dot(const Frag &a, const Frag &b) {
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) s = __builtin_fmaf((float)a[c][e], (float)b[c][e], s);
    return s;
  }
  __device__ __forceinline__ void rows_times(const char *blk, const Frag &f, f32x16 &acc) const {
    acc = f32x16{};
#pragma unroll
    for (int c = 0; c < NCH; ++c)
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(blk + row[c]), f[c], acc, 0, 0, 0);
  }
  // (the weights are rounded to bf16 as the matrix cores' operand)
  __device__ __forceinline__ void cols_times(const char *blk, const f32x16 &w, f32x16 (&acc)[NDB]) const {
    bf16x8 x[2];
#pragma unroll
    for (int v = 0; v < 16; ++v) x[v >> 3][v & 7] = (__bf16)w[v];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int db = 0; db < NDB; ++db)
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_read_tr16x2(blk + tr[db] + 16 * t * ROW, ROW), x[t],
                                                          acc[db], 0, 0, 0);
  }
  // f(column, four consecutive values) over a lane's slots
  template <class F>
  static __device__ __forceinline__ void columns(const f32x16 (&acc)[NDB], int half, F f) {
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        f(32 * db + 8 * g + 4 * half, f32x4{acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]});
  }
};

template <int D>
struct Tile<float, D> {
  static constexpr int ROW = D * 4, CPR = D / 4, NDB = D / 32, NCH = D / 8;
  typedef f32x4 Frag[NCH];
  int row[NCH];   // by rows: chunk c of this lane's row
  int colm[4];    // by columns: rows 8 half + r, r % 4 = index

  static __device__ __forceinline__ int swz(int r) { return swz_f32(r); }
  __device__ __forceinline__ void init(int lane) {
    const int col = lane & 31, half = lane >> 5, r = row_perm(col);
#pragma unroll
    for (int c = 0; c < NCH; ++c) row[c] = r * ROW + (((half * NCH + c) ^ swz(r)) * 16);
    const int e = col * NDB;   // first column
#pragma unroll
    for (int i = 0; i < 4; ++i) colm[i] = 8 * half * ROW + (((e >> 2) ^ (i | (half << 2))) * 16) + (e & 3) * 4;
  }
  static __device__ __forceinline__ void load(Frag &f, const float *p, int half) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) f[c] = *reinterpret_cast<const f32x4 *>(p + half * (D / 2) + 4 * c);
  }
  static __device__ __forceinline__ float dot(const Frag &a, const Frag &b) {
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_fmaf(a[c][e], b[c][e], s);
    return s;
  }
  __device__ __forceinline__ void rows_times(const char *blk, const Frag &f, f32x16 &acc) const {
    mfma_rows_f32<NCH, 4>(blk, row, f, acc);
  }
  __device__ __forceinline__ void cols_times(const char *blk, const f32x16 &w, f32x16 (&acc)[NDB]) const {
    mfma_cols_f32<NDB>([&](int t) { return blk + colm[t & 3] + (16 * (t >> 3) + (t & 7)) * ROW; }, w, acc);
  }
  template <class F>
  static __device__ __forceinline__ void columns(const f32x16 (&acc)[NDB], int half, F f) {
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int x = 0; x < NDB; ++x) {   // the accumulators' columns alternate
        f32x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = acc[(4 * x + i) % NDB][4 * g + (4 * x + i) / NDB];
        f(NDB * (8 * g + 4 * half) + 4 * x, o);
      }
  }
};

// Four consecutive values as T.
template <typename T>
__device__ __forceinline__ void put4(T *p, const f32x4 &v) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<f32x4 *>(p) = v;
  } else {
    bf16x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (__bf16)v[e];
    *reinterpret_cast<bf16x4 *>(p) = o;
  }
}

// One wave's 32 rows from accumulators (this lane's row `col`) to memory, through a
// staging area of 32 * (ROW + 16) bytes of its own so that the stores cover whole
// rows. at(r): row r's address, NULL to leave it out. The wave's own LDS operations
// are in order, so no barrier is needed.
template <typename T, int D, class At>
__device__ __forceinline__ void store_rows(char *area, const f32x16 (&acc)[D / 32], float mul, int lane, At at) {
  using Tl = Tile<T, D>;
  constexpr int PITCH = Tl::ROW + 16;
  T *mine = reinterpret_cast<T *>(area + (lane & 31) * PITCH);
  Tl::columns(acc, lane >> 5, [&](int c, f32x4 v) { put4<T>(mine + c, v * mul); });
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
  for (int k = 0; k < 32 * Tl::CPR / 64; ++k) {
    const int i = lane + 64 * k, r = i / Tl::CPR, c = i % Tl::CPR;
    T *dst = at(r);
    if (dst) reinterpret_cast<uint4 *>(dst)[c] = *reinterpret_cast<const uint4 *>(area + r * PITCH + c * 16);
  }
}

}  // namespace hla
