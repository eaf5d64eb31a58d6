// Argument checks shared by the C-ABI entry points. A failed check leaves its text
// for hla_last_error() on the calling thread and returns the status.
#pragma once

#include "hla_internal.h"

namespace hla {

hla_status fail(hla_status st, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

inline hla_status hip_status(hipError_t e, const char *what) {
  if (e == hipSuccess) return HLA_OK;
  return fail(HLA_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

inline bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline bool is_pow2(int64_t x) { return x > 0 && (x & (x - 1)) == 0; }
inline int64_t dtype_size(hla_dtype dt) { return dt == HLA_F32 ? 4 : (dt == HLA_BF16 ? 2 : 0); }

constexpr int64_t kMaxI32 = 2147483647LL;

inline hla_status check_tensor_args(const void *a, const char *name) {
  if (!a) return fail(HLA_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned(a, 16)) return fail(HLA_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
  return HLA_OK;
}

inline bool overlaps(const void *a, int64_t na, const void *b, int64_t nb) {
  const char *x = static_cast<const char *>(a), *y = static_cast<const char *>(b);
  return x < y + nb && y < x + na;
}

// A strided [B, heads, N, d] tensor of one call, sizes and element size included.
struct ViewShape {
  const char *name;
  hla_view v;
  int64_t size[3];    // B, heads, N
  int64_t d, es;
  int64_t stride(int i) const { return i == 0 ? v.batch : (i == 1 ? v.head : v.row); }
  // bytes from the first element to the end of the last
  int64_t extent() const {
    int64_t n = d;
    for (int i = 0; i < 3; ++i) n += (size[i] - 1) * stride(i);
    return n * es;
  }
};

// Pointer, alignment and strides of a view; written: its rows must not overlap each
// other. Strides of dimensions of size 1 are not looked at (and set to 0).
hla_status check_view(ViewShape &s, bool written);
// Whether two views may share an element. Views whose address ranges meet are told
// apart where they interleave, as the q, k and v rows of one tensor do.
bool views_clash(const ViewShape &a, const ViewShape &b);
// Whether a view may share an element with n bytes at p.
inline bool view_clash(const ViewShape &a, const void *p, int64_t n) {
  return overlaps(a.v.ptr, a.extent(), p, n);
}

}  // namespace hla
