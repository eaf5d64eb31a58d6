// C-ABI entry points of the operators around the attention in a transformer block:
// argument validation on the host, then launch. As in hla_api.cpp every check runs
// before the first HIP call.
#include <algorithm>
#include <cmath>
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
