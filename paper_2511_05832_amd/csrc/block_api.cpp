// C-ABI entry points of the operators around the attention in a transformer block:
// argument validation on the host, then launch. Every check but the workspace's runs before
// the first HIP call; how large that has to be depends on the device, so the device is asked
// for its size (nothing else) before those last checks. Nothing is enqueued before all pass.
#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <utility>

#include "api_common.h"

namespace hla {

hla_status check_view(ViewShape &s, bool written) {
  hla_status st = check_tensor_args(s.v.ptr, s.name);
  if (st != HLA_OK) return st;
  int64_t *strides[3] = {&s.v.batch, &s.v.head, &s.v.row};
  const int64_t most = (1LL << 46) / s.es;
  for (int i = 0; i < 3; ++i) {
    if (s.size[i] == 1) *strides[i] = 0;
    if (*strides[i] < 0 || *strides[i] > most || *strides[i] * s.es % 16)
      return fail(HLA_ERR_INVALID_ARG, "%s: stride %lld must be >= 0 and a multiple of 16 bytes", s.name,
                  (long long)*strides[i]);
    if (*strides[i] && s.size[i] - 1 > most / *strides[i])
      return fail(HLA_ERR_UNSUPPORTED, "%s reaches over more than 2^46 bytes", s.name);
  }
  if (!written) return HLA_OK;
  // from the innermost stride out, each must step over all that lies within it
  std::pair<int64_t, int64_t> dims[3];   // stride, size
  for (int i = 0; i < 3; ++i) dims[i] = {*strides[i], s.size[i]};
  std::sort(dims, dims + 3);
  int64_t span = s.d;
  for (const auto &e : dims) {
    if (e.second == 1) continue;
    if (e.first < span) return fail(HLA_ERR_INVALID_ARG, "the rows of %s overlap each other", s.name);
    span += (e.second - 1) * e.first;
  }
  return HLA_OK;
}

// Two views whose ranges meet share no element if, for some stride c, the strides of
// either that reach over c are multiples of it and what lies within c (the elements
// of the others) falls on separate parts of every period of c.
bool views_clash(const ViewShape &a, const ViewShape &b) {
  if (!overlaps(a.v.ptr, a.extent(), b.v.ptr, b.extent())) return false;
  const ViewShape &lo = a.v.ptr <= b.v.ptr ? a : b, &hi = a.v.ptr <= b.v.ptr ? b : a;
  const int64_t bytes = static_cast<const char *>(hi.v.ptr) - static_cast<const char *>(lo.v.ptr);
  if (bytes % a.es) return true;
  const int64_t delta = bytes / a.es;
  for (const ViewShape *t : {&lo, &hi})
    for (int i = 0; i < 3; ++i) {
      const int64_t c = t->stride(i);
      if (c <= 0) continue;
      int64_t span[2];
      int n = 0;
      for (const ViewShape *x : {&lo, &hi}) {
        int64_t w = x->d;
        for (int j = 0; j < 3; ++j)
          if (x->stride(j) % c) w += (x->size[j] - 1) * x->stride(j);
        span[n++] = w;
      }
      const int64_t at = delta % c;
      if (at >= span[0] && at + span[1] <= c) return false;
    }
  return true;
}

}  // namespace hla

using namespace hla;

namespace {

bool same_view(const ViewShape &a, const ViewShape &b) {
  return a.v.ptr == b.v.ptr && a.v.batch == b.v.batch && a.v.head == b.v.head && a.v.row == b.v.row;
}

RopeTensor rope_tensor(const ViewShape &s) { return {s.v.ptr, s.v.batch, s.v.head, s.v.row}; }

}  // namespace

extern "C" {

hla_status hla_rope(const hla_view *q, const hla_view *k, const hla_view *q_out,
                    const hla_view *k_out, const int32_t *pos, int64_t pos_stride,
                    const double *freqs, int64_t B, int64_t heads, int64_t kv_heads, int64_t N,
                    int64_t d, int64_t pairs, int32_t grid_w, int32_t interleaved,
                    int32_t inverse, float magnitude, hla_dtype dtype, hla_stream_t stream) {
  hla_status st;
  const int64_t es = dtype_size(dtype);
  if (!es) return fail(HLA_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
  if (!q || !q_out) return fail(HLA_ERR_INVALID_ARG, "q or q_out is NULL");
  if ((k != nullptr) != (k_out != nullptr)) return fail(HLA_ERR_INVALID_ARG, "give k and k_out, or neither");
  const int nt = k ? 2 : 1;
  if (!k) kv_heads = 0;
  if (B <= 0 || heads <= 0 || N <= 0 || d <= 0 || pairs <= 0 || kv_heads < 0 || (k && kv_heads == 0))
    return fail(HLA_ERR_INVALID_ARG, "sizes must be positive");
  if (grid_w < 0) return fail(HLA_ERR_INVALID_ARG, "grid_w = %d must be >= 0", grid_w);
  if (!std::isfinite(magnitude)) return fail(HLA_ERR_INVALID_ARG, "magnitude must be finite");
  const int axes = grid_w ? 2 : 1;
  if (pairs > d || 2 * pairs * axes > d)
    return fail(HLA_ERR_INVALID_ARG, "%lld features are turned, a row has %lld", (long long)(2 * pairs * axes),
                (long long)d);
  if (d > (1 << 20) || d * es % 16) return fail(HLA_ERR_UNSUPPORTED, "row of %lld bytes is not a multiple of 16", (long long)(d * es));
  if (B > kMaxI32 || heads > (1 << 20) || kv_heads > (1 << 20) || N > (1LL << 30) || B * (heads + kv_heads) > (1LL << 30) ||
      N * (d / 2) > (1LL << 30) / B)
    return fail(HLA_ERR_UNSUPPORTED, "B * N * d / 2 exceeds 2^30, or B * heads does");
  if (!freqs) return fail(HLA_ERR_INVALID_ARG, "freqs is NULL");
  if (!aligned(freqs, 8)) return fail(HLA_ERR_INVALID_ARG, "freqs is not 8-byte aligned");
  if (pos && !aligned(pos, 4)) return fail(HLA_ERR_INVALID_ARG, "pos is not 4-byte aligned");
  if (pos && pos_stride != 0 && (pos_stride < N || pos_stride > (1LL << 40)))
    return fail(HLA_ERR_INVALID_ARG, "pos_stride = %lld must be 0 or at least N", (long long)pos_stride);
  if (!pos) pos_stride = 0;
  ViewShape in[2] = {{"q", *q, {B, heads, N}, d, es}, {"k", k ? *k : *q, {B, kv_heads, N}, d, es}};
  ViewShape out[2] = {{"q_out", *q_out, {B, heads, N}, d, es}, {"k_out", k ? *k_out : *q_out, {B, kv_heads, N}, d, es}};
  for (int i = 0; i < nt; ++i) {
    if ((st = check_view(in[i], false)) != HLA_OK) return st;
    if ((st = check_view(out[i], true)) != HLA_OK) return st;
  }
  const int64_t pos_bytes = ((pos_stride ? (B - 1) * pos_stride : 0) + N) * 4;
  for (int i = 0; i < nt; ++i) {
    for (int j = 0; j < nt; ++j)
      if (!(i == j && same_view(in[j], out[i])) && views_clash(in[j], out[i]))
        return fail(HLA_ERR_INVALID_ARG, "%s overlaps %s", out[i].name, in[j].name);
    if (pos && view_clash(out[i], pos, pos_bytes)) return fail(HLA_ERR_INVALID_ARG, "%s overlaps pos", out[i].name);
    if (view_clash(out[i], freqs, pairs * 8)) return fail(HLA_ERR_INVALID_ARG, "%s overlaps freqs", out[i].name);
  }
  if (nt == 2 && views_clash(out[0], out[1])) return fail(HLA_ERR_INVALID_ARG, "q_out overlaps k_out");
  RopeArgs a;
  for (int i = 0; i < 2; ++i) {
    a.in[i] = rope_tensor(in[i < nt ? i : 0]);
    a.out[i] = rope_tensor(out[i < nt ? i : 0]);
  }
  a.pos = pos;
  a.pos_stride = pos_stride;
  a.freqs = freqs;
  a.B = (int32_t)B;
  a.heads[0] = (int32_t)heads;
  a.heads[1] = (int32_t)kv_heads;
  a.N = (int32_t)N;
  a.d = (int32_t)d;
  a.pairs = (int32_t)pairs;
  a.axes = axes;
  a.grid_w = grid_w;
  a.interleaved = interleaved != 0;
  a.inverse = inverse != 0;
  a.magnitude = magnitude;
  return hip_status(launch_rope(a, dtype, (hipStream_t)stream), "hla_rope");
}

}  // extern "C"

namespace {

CrossStride cross_stride(const ViewShape &s) {
  return {s.v.batch * s.es, (uint32_t)(s.v.head * s.es / 16), (uint32_t)(s.v.row * s.es / 16)};
}

// A launch counts its threads in 32 bits: below 2^24 workgroups of 256 (of 512, half as
// many, which are counted twice), the rounding of their number included.
constexpr int64_t kMostGroups = (1 << 24) - 512;

// Sizes of a cross attention, into the kernel's arguments.
hla_status cross_sizes(int64_t B, int64_t heads, int64_t kv_heads, int64_t N, int64_t M, int64_t d,
                       hla_dtype dtype, bool backward, CrossArgs *a) {
  if (!dtype_size(dtype)) return fail(HLA_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
  if (B <= 0 || heads <= 0 || kv_heads <= 0 || N <= 0 || M <= 0 || d <= 0)
    return fail(HLA_ERR_INVALID_ARG, "sizes must be positive");
  if (heads % kv_heads)
    return fail(HLA_ERR_INVALID_ARG, "heads = %lld must be a multiple of kv_heads = %lld", (long long)heads, (long long)kv_heads);
  if (d != 32 && d != 64) return fail(HLA_ERR_UNSUPPORTED, "head_dim %lld (supported: 32, 64)", (long long)d);
  const int64_t G = heads / kv_heads, most = 1LL << 30;
  if (B > most || heads > most || N > most || M > most || G > most / N || B > most / kv_heads)
    return fail(HLA_ERR_UNSUPPORTED, "heads / kv_heads * N, M or B * kv_heads exceeds 2^30");
  const int64_t bk = B * kv_heads, R = G * N;
  if (M > (1LL << 36) / bk) return fail(HLA_ERR_UNSUPPORTED, "B * kv_heads * M exceeds 2^36");
  if (bk * ((R + 127) / 128) > kMostGroups || (backward && 2 * bk * ((M + 127) / 128) > kMostGroups))
    return fail(HLA_ERR_UNSUPPORTED, "B * kv_heads times the tiles of 128 rows, or twice those of 128 keys, is not below 2^24 - 2^9");
  a->B = (int32_t)B;
  a->heads = (int32_t)heads;
  a->kv = (int32_t)kv_heads;
  a->G = (int32_t)G;
  a->N = (int32_t)N;
  a->M = (int32_t)M;
  a->R = (int32_t)R;
  a->Rp = (int32_t)((R + 127) / 128 * 128);
  a->ndiv = make_fastdiv((uint32_t)N);
  return HLA_OK;
}

// How the work is shared out on the current device; returns the bytes of workspace.
int64_t cross_plan(CrossArgs &a, int64_t d, hla_dtype dtype, bool backward) {
  const int64_t es = dtype_size(dtype), bk = (int64_t)a.B * a.kv;
  if (!backward) return cross_fwd_plan(a, (int)(d * es)) ? bk * a.splits * a.R * (4 * d + 8) : 0;
  const bool parts = cross_bwd_plan(a, (int)d, (int)es);
  return 8 * bk * a.Rp + (parts ? ((int64_t)a.pieces << a.kshift) * 8 * d : 0);
}

hla_status cross_scale(float scale, CrossArgs *a) {
  if (!(scale > 0.f) || scale > 1e30f) return fail(HLA_ERR_INVALID_ARG, "scale must be positive and finite");
  a->scale = scale;
  a->scale_log2 = (float)((double)scale * 1.4426950408889634074);
  return HLA_OK;
}

// Views (q, k, v first, outputs last): pointers and strides of each, and no output on
// another view or on one of the plain ranges.
struct Range {
  const char *name;
  const void *p;
  int64_t bytes;
  bool given() const { return p && bytes; }
};
typedef std::initializer_list<Range> Ranges;
hla_status cross_views(ViewShape *t, int n_in, int n, Ranges ranges) {
  hla_status st;
  for (int i = 0; i < n; ++i)
    if ((st = check_view(t[i], i >= n_in)) != HLA_OK) return st;
  for (int i = 0; i < n; ++i)
    if (((t[i].size[1] - 1) * t[i].v.head + (t[i].size[2] - 1) * t[i].v.row) * t[i].es >= (1LL << 36))
      return fail(HLA_ERR_UNSUPPORTED, "a batch element of %s reaches over 2^36 bytes", t[i].name);
  for (int i = 1; i < 3; ++i)   // k, v
    if (t[i].v.row * t[i].es >= (1 << 25))
      return fail(HLA_ERR_UNSUPPORTED, "the rows of %s must lie less than 2^25 bytes apart", t[i].name);
  for (int i = n_in; i < n; ++i)
    for (int j = 0; j < i; ++j)
      if (views_clash(t[i], t[j])) return fail(HLA_ERR_INVALID_ARG, "%s overlaps %s", t[i].name, t[j].name);
  for (const Range &r : ranges)
    for (int i = n_in; i < n; ++i)
      if (r.given() && view_clash(t[i], r.p, r.bytes))
        return fail(HLA_ERR_INVALID_ARG, "%s overlaps %s", t[i].name, r.name);
  return HLA_OK;
}

// The workspace, which lies on none of them.
hla_status cross_work(int64_t need, const void *work, int64_t bytes, const ViewShape *t, int n_in, int n, Ranges ranges) {
  if (!need) return HLA_OK;
  if (!work) return fail(HLA_ERR_INVALID_ARG, "work is NULL, %lld bytes are needed", (long long)need);
  if (!aligned(work, 16)) return fail(HLA_ERR_INVALID_ARG, "work is not 16-byte aligned");
  if (bytes < need)
    return fail(HLA_ERR_INVALID_ARG, "work has %lld bytes, %lld are needed", (long long)bytes, (long long)need);
  for (int i = 0; i < n; ++i)
    if (view_clash(t[i], work, need))
      return i < n_in ? fail(HLA_ERR_INVALID_ARG, "work overlaps %s", t[i].name)
                      : fail(HLA_ERR_INVALID_ARG, "%s overlaps work", t[i].name);
  for (const Range &r : ranges)
    if (r.given() && overlaps(r.p, r.bytes, work, need)) return fail(HLA_ERR_INVALID_ARG, "work overlaps %s", r.name);
  return HLA_OK;
}

}  // namespace

extern "C" {

hla_status hla_cross_attn_workspace(int64_t B, int64_t heads, int64_t kv_heads, int64_t N,
                                    int64_t M, int64_t d, hla_dtype dtype, int32_t backward,
                                    int64_t *bytes) {
  CrossArgs a;
  if (!bytes) return fail(HLA_ERR_INVALID_ARG, "bytes is NULL");
  hla_status st = cross_sizes(B, heads, kv_heads, N, M, d, dtype, backward != 0, &a);
  if (st != HLA_OK) return st;
  *bytes = cross_plan(a, d, dtype, backward != 0);
  return HLA_OK;
}

hla_status hla_cross_attn_fwd(const hla_view *q, const hla_view *k, const hla_view *v,
                              const int32_t *lengths, const hla_view *out, float *lse, int64_t B,
                              int64_t heads, int64_t kv_heads, int64_t N, int64_t M, int64_t d,
                              hla_dtype dtype, float scale, void *work, int64_t work_bytes,
                              hla_stream_t stream) {
  hla_status st;
  CrossArgs a = {};
  if (!q || !k || !v || !out) return fail(HLA_ERR_INVALID_ARG, "q, k, v or out is NULL");
  if ((st = cross_sizes(B, heads, kv_heads, N, M, d, dtype, false, &a)) != HLA_OK) return st;
  if ((st = cross_scale(scale, &a)) != HLA_OK) return st;
  if (lse && !aligned(lse, 4)) return fail(HLA_ERR_INVALID_ARG, "lse is not 4-byte aligned");
  if (lengths && !aligned(lengths, 4)) return fail(HLA_ERR_INVALID_ARG, "lengths is not 4-byte aligned");
  const int64_t es = dtype_size(dtype), lse_bytes = lse ? B * heads * N * 4 : 0;
  ViewShape t[4] = {{"q", *q, {B, heads, N}, d, es}, {"k", *k, {B, kv_heads, M}, d, es},
                    {"v", *v, {B, kv_heads, M}, d, es}, {"out", *out, {B, heads, N}, d, es}};
  const Ranges ranges = {{"lse", lse, lse_bytes}, {"lengths", lengths, B * 4}};
  if ((st = cross_views(t, 3, 4, ranges)) != HLA_OK) return st;
  for (int i = 0; i < 3; ++i)
    if (lse && view_clash(t[i], lse, lse_bytes)) return fail(HLA_ERR_INVALID_ARG, "lse overlaps %s", t[i].name);
  if (lse && lengths && overlaps(lse, lse_bytes, lengths, B * 4)) return fail(HLA_ERR_INVALID_ARG, "lse overlaps lengths");
  const int64_t need = cross_plan(a, d, dtype, false);
  if ((st = cross_work(need, work, work_bytes, t, 3, 4, ranges)) != HLA_OK) return st;
  a.q = t[0].v.ptr;
  a.k = t[1].v.ptr;
  a.v = t[2].v.ptr;
  a.out = t[3].v.ptr;
  a.qs = cross_stride(t[0]);
  a.ks = cross_stride(t[1]);
  a.vs = cross_stride(t[2]);
  a.os = cross_stride(t[3]);
  a.lse = lse;
  a.lengths = lengths;
  if (need) {
    a.part = static_cast<float *>(work);
    a.part_ml = reinterpret_cast<float2 *>(a.part + (int64_t)a.B * a.kv * a.splits * a.R * d);
  }
  return hip_status(launch_cross_fwd(a, (int)d, dtype, (hipStream_t)stream), "hla_cross_attn_fwd");
}

hla_status hla_cross_attn_bwd(const hla_view *q, const hla_view *k, const hla_view *v,
                              const hla_view *out, const hla_view *dout, const float *lse,
                              const int32_t *lengths, const hla_view *dq, const hla_view *dk,
                              const hla_view *dv, int64_t B, int64_t heads, int64_t kv_heads,
                              int64_t N, int64_t M, int64_t d, hla_dtype dtype, float scale,
                              void *work, int64_t work_bytes, hla_stream_t stream) {
  hla_status st;
  CrossArgs a = {};
  if (!q || !k || !v || !out || !dout || !dq || !dk || !dv) return fail(HLA_ERR_INVALID_ARG, "a tensor is NULL");
  if ((st = cross_sizes(B, heads, kv_heads, N, M, d, dtype, true, &a)) != HLA_OK) return st;
  if ((st = cross_scale(scale, &a)) != HLA_OK) return st;
  if (!lse) return fail(HLA_ERR_INVALID_ARG, "lse is NULL");
  if (!aligned(lse, 4)) return fail(HLA_ERR_INVALID_ARG, "lse is not 4-byte aligned");
  if (lengths && !aligned(lengths, 4)) return fail(HLA_ERR_INVALID_ARG, "lengths is not 4-byte aligned");
  const int64_t es = dtype_size(dtype), lse_bytes = B * heads * N * 4;
  ViewShape t[8] = {{"q", *q, {B, heads, N}, d, es},       {"k", *k, {B, kv_heads, M}, d, es},
                    {"v", *v, {B, kv_heads, M}, d, es},    {"out", *out, {B, heads, N}, d, es},
                    {"dout", *dout, {B, heads, N}, d, es}, {"dq", *dq, {B, heads, N}, d, es},
                    {"dk", *dk, {B, kv_heads, M}, d, es},  {"dv", *dv, {B, kv_heads, M}, d, es}};
  const Ranges ranges = {{"lse", lse, lse_bytes}, {"lengths", lengths, B * 4}};
  if ((st = cross_views(t, 5, 8, ranges)) != HLA_OK) return st;
  const int64_t need = cross_plan(a, d, dtype, true);
  if ((st = cross_work(need, work, work_bytes, t, 5, 8, ranges)) != HLA_OK) return st;
  a.q = t[0].v.ptr;
  a.k = t[1].v.ptr;
  a.v = t[2].v.ptr;
  a.out = t[3].v.ptr;
  a.dout = t[4].v.ptr;
  a.dq = t[5].v.ptr;
  a.dk = t[6].v.ptr;
  a.dv = t[7].v.ptr;
  a.qs = cross_stride(t[0]);
  a.ks = cross_stride(t[1]);
  a.vs = cross_stride(t[2]);
  a.os = cross_stride(t[3]);
  a.gs = cross_stride(t[4]);
  a.dqs = cross_stride(t[5]);
  a.dks = cross_stride(t[6]);
  a.dvs = cross_stride(t[7]);
  a.lse = const_cast<float *>(lse);
  a.lengths = lengths;
  a.stats = static_cast<float *>(work);
  a.part = a.stats + 2 * (int64_t)a.B * a.kv * a.Rp;
  return hip_status(launch_cross_bwd(a, (int)d, dtype, (hipStream_t)stream), "hla_cross_attn_bwd");
}

}  // extern "C"

namespace {

struct Tensor {
  const char *name;
  const void *p;
  int64_t bytes;
};

hla_status linear_sizes(int64_t T, int64_t K, int64_t F, hla_act act, hla_dtype dtype, bool backward, LinearArgs *a) {
  const int64_t es = dtype_size(dtype);
  if (!es) return fail(HLA_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
  if (act < HLA_ACT_NONE || act > HLA_ACT_SILU) return fail(HLA_ERR_INVALID_ARG, "unknown activation %d", (int)act);
  if (T <= 0 || K <= 0 || F <= 0) return fail(HLA_ERR_INVALID_ARG, "sizes must be positive");
  if (K * es % 16 || F * es % 16)
    return fail(HLA_ERR_UNSUPPORTED, "K = %lld and F = %lld must be multiples of %lld", (long long)K, (long long)F,
                (long long)(16 / es));
  if (T > (1LL << 30) || K >= (1 << 20) || F >= (1 << 20))
    return fail(HLA_ERR_UNSUPPORTED, "T above 2^30, or K or F not below 2^20");
  // (a launch counts its threads in 32 bits: below 2^24 workgroups of 256, one to a tile of
  // 64 x 64; larger tiles have up to 512 threads, and are at most half as many)
  const int64_t t = (T + 63) / 64, k = (K + 63) / 64, f = (F + 63) / 64, most = (1 << 24) - 4;
  if (t * std::max(k, f) > most || (backward && k * f > most))
    return fail(HLA_ERR_UNSUPPORTED, "T * max(K, F), or K * F of a backward, in tiles of 64 x 64, is not below 2^36");
  *a = {};
  a->T = (int32_t)T;
  a->K = (int32_t)K;
  a->F = (int32_t)F;
  a->act = act;
  return HLA_OK;
}

// The inputs' and outputs' pointers, and no output on an input or another output. NULL
// entries are left out.
hla_status linear_tensors(const Tensor *in, int ni, const Tensor *out, int no) {
  hla_status st;
  for (int i = 0; i < ni; ++i)
    if (in[i].p && (st = check_tensor_args(in[i].p, in[i].name)) != HLA_OK) return st;
  for (int i = 0; i < no; ++i) {
    if (!out[i].p) continue;
    if ((st = check_tensor_args(out[i].p, out[i].name)) != HLA_OK) return st;
    for (int j = 0; j < ni; ++j)
      if (in[j].p && overlaps(out[i].p, out[i].bytes, in[j].p, in[j].bytes))
        return fail(HLA_ERR_INVALID_ARG, "%s overlaps %s", out[i].name, in[j].name);
    for (int j = 0; j < i; ++j)
      if (out[j].p && overlaps(out[i].p, out[i].bytes, out[j].p, out[j].bytes))
        return fail(HLA_ERR_INVALID_ARG, "%s overlaps %s", out[i].name, out[j].name);
  }
  return HLA_OK;
}

// The workspace, which lies on none of them.
hla_status linear_work(const Tensor *in, int ni, const Tensor *out, int no, const void *work, int64_t need) {
  if (!aligned(work, 16)) return fail(HLA_ERR_INVALID_ARG, "work is not 16-byte aligned");
  for (const auto &list : {std::make_pair(in, ni), std::make_pair(out, no)})
    for (int i = 0; i < list.second; ++i)
      if (list.first[i].p && overlaps(work, need, list.first[i].p, list.first[i].bytes))
        return fail(HLA_ERR_INVALID_ARG, "work overlaps %s", list.first[i].name);
  return HLA_OK;
}

}  // namespace

extern "C" {

hla_status hla_linear(const void *x, const void *w, const void *bias, const void *residual,
                      hla_act act, void *y, void *pre, int64_t T, int64_t K, int64_t F,
                      hla_dtype dtype, void *work, int64_t work_bytes, hla_stream_t stream) {
  LinearArgs a;
  hla_status st = linear_sizes(T, K, F, act, dtype, false, &a);
  if (st != HLA_OK) return st;
  if (!x || !w || !y) return fail(HLA_ERR_INVALID_ARG, "%s is NULL", !x ? "x" : (!w ? "w" : "y"));
  const int64_t es = dtype_size(dtype);
  // (residual == y is allowed: each element is read before it is written, by one thread)
  const Tensor in[4] = {{"x", x, T * K * es}, {"w", w, F * K * es}, {"bias", bias, F * es},
                        {"residual", residual == y ? nullptr : residual, T * F * es}};
  const Tensor out[2] = {{"y", y, T * F * es}, {"pre", pre, T * F * es}};
  if ((st = linear_tensors(in, 4, out, 2)) != HLA_OK) return st;
  a.parts = true;
  const int64_t need = linear_fwd_work(a, dtype);
  a.parts = need > 0 && work && work_bytes >= need;
  if (a.parts && (st = linear_work(in, 4, out, 2, work, need)) != HLA_OK) return st;
  a.work = work;
  a.x = x;
  a.w = w;
  a.bias = bias;
  a.residual = residual;
  a.y = y;
  a.pre = pre;
  return hip_status(launch_linear(a, dtype, (hipStream_t)stream), "hla_linear");
}

hla_status hla_linear_workspace(int64_t T, int64_t K, int64_t F, hla_act act, hla_dtype dtype,
                                int32_t backward, int64_t *bytes) {
  LinearArgs a;
  if (!bytes) return fail(HLA_ERR_INVALID_ARG, "bytes is NULL");
  hla_status st = linear_sizes(T, K, F, act, dtype, backward != 0, &a);
  if (st != HLA_OK) return st;
  a.dx = a.dw = a.db = bytes;   // (all of them; the addresses are not used)
  a.parts = true;
  *bytes = backward ? linear_bwd_work(a, dtype).bytes : linear_fwd_work(a, dtype);
  return HLA_OK;
}

hla_status hla_linear_bwd(const void *x, const void *w, const void *pre, const void *dy,
                          hla_act act, void *dx, void *dw, void *db, int64_t T, int64_t K,
                          int64_t F, hla_dtype dtype, void *work, int64_t work_bytes,
                          hla_stream_t stream) {
  LinearArgs a;
  hla_status st = linear_sizes(T, K, F, act, dtype, true, &a);
  if (st != HLA_OK) return st;
  if (!dx && !dw && !db) return fail(HLA_ERR_INVALID_ARG, "dx, dw and db are all NULL");
  if (!dy) return fail(HLA_ERR_INVALID_ARG, "dy is NULL");
  if (dx && !w) return fail(HLA_ERR_INVALID_ARG, "w is NULL");
  if (dw && !x) return fail(HLA_ERR_INVALID_ARG, "x is NULL");
  if (act != HLA_ACT_NONE && !pre) return fail(HLA_ERR_INVALID_ARG, "pre is NULL");
  if (act == HLA_ACT_NONE) pre = nullptr;
  a.x = x;
  a.w = w;
  a.pre = const_cast<void *>(pre);
  a.dy = dy;
  a.dx = dx;
  a.dw = dw;
  a.db = db;
  const int64_t es = dtype_size(dtype);
  const Tensor in[4] = {{"x", x, T * K * es}, {"w", w, F * K * es}, {"pre", pre, T * F * es}, {"dy", dy, T * F * es}};
  const Tensor out[3] = {{"dx", dx, T * K * es}, {"dw", dw, F * K * es}, {"db", db, F * es}};
  if ((st = linear_tensors(in, 4, out, 3)) != HLA_OK) return st;
  const int64_t need = linear_bwd_work(a, dtype).bytes;
  if (need && !work) return fail(HLA_ERR_INVALID_ARG, "work is NULL, %lld bytes are needed", (long long)need);
  if (work_bytes < need)
    return fail(HLA_ERR_INVALID_ARG, "work has %lld bytes, %lld are needed", (long long)work_bytes, (long long)need);
  if (need && (st = linear_work(in, 4, out, 3, work, need)) != HLA_OK) return st;
  a.work = work;
  return hip_status(launch_linear_bwd(a, dtype, (hipStream_t)stream), "hla_linear_bwd");
}

}  // extern "C"
