// Argument checks shared by the entry points (host code).
#pragma once
#include <stdint.h>

#include "tokenring.h"

namespace tr {

// Records the message for tr_last_error() and returns the status; clear_error() empties it (both defined in api.hip).
tr_status fail(tr_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
void clear_error();

inline int64_t elem_bytes(int32_t dtype) { return dtype == TR_BF16 ? 2 : dtype == TR_F32 ? 4 : 1; }

// Number of elements from ptr to one past the last addressed element of the view.
inline int64_t extent_elems(const tr_tensor* t) {
  if (t->B == 0 || t->H == 0 || t->S == 0 || t->D == 0) return 0;
  return (t->B - 1) * t->stride_b + (t->H - 1) * t->stride_h + (t->S - 1) * t->stride_s + t->D;
}

inline bool overlaps(const tr_tensor* a, const tr_tensor* b) {
  const int64_t ea = extent_elems(a) * elem_bytes(a->dtype), eb = extent_elems(b) * elem_bytes(b->dtype);
  if (ea == 0 || eb == 0) return false;
  const uintptr_t a0 = (uintptr_t)a->ptr, b0 = (uintptr_t)b->ptr;
  return a0 < b0 + (uintptr_t)eb && b0 < a0 + (uintptr_t)ea;
}

// Types that an argument may have, one bit each.
constexpr unsigned kBf16 = 1u << TR_BF16, kF32 = 1u << TR_F32, kF8 = 1u << TR_F8E4M3, kE8m0 = 1u << TR_F8E8M0;

// Common checks of one descriptor. `row_align` = required multiple (in elements) of the strides
// and byte alignment of the pointer for vector access.
inline tr_status check_typed(const char* name, const tr_tensor* t, unsigned types, int row_align_bytes) {
  static const char* const names[] = {"bf16", "fp32", "e4m3", "e8m0"};
  if (!t) return fail(TR_ERR_NULL, "%s: descriptor is NULL", name);
  if (t->dtype < TR_BF16 || t->dtype > TR_F8E8M0) return fail(TR_ERR_DTYPE, "%s: unknown dtype %d", name, (int)t->dtype);
  if (!(types >> t->dtype & 1)) return fail(TR_ERR_DTYPE, "%s: dtype %s not supported for this argument", name, names[t->dtype]);
  if (t->B < 0 || t->H < 0 || t->S < 0 || t->D < 0) return fail(TR_ERR_SHAPE, "%s: negative dimension", name);
  if (t->B > INT32_MAX || t->H > INT32_MAX || t->S > (1 << 30) || t->D > INT32_MAX)
    return fail(TR_ERR_SHAPE, "%s: dimension too large", name);
  const bool empty = extent_elems(t) == 0;
  if (!empty && !t->ptr) return fail(TR_ERR_NULL, "%s: data pointer is NULL", name);
  if (t->stride_b < 0 || t->stride_h < 0 || t->stride_s < 0) return fail(TR_ERR_STRIDE, "%s: negative stride", name);
  if (!empty) {
    if (t->S > 1 && t->stride_s < t->D) return fail(TR_ERR_STRIDE, "%s: stride_s %lld smaller than D %lld", name, (long long)t->stride_s, (long long)t->D);
    const int64_t eb = elem_bytes(t->dtype);
    if (row_align_bytes > 1) {
      if (((uintptr_t)t->ptr) % row_align_bytes) return fail(TR_ERR_STRIDE, "%s: pointer not %d-byte aligned", name, row_align_bytes);
      if ((t->stride_b * eb) % row_align_bytes || (t->stride_h * eb) % row_align_bytes || (t->stride_s * eb) % row_align_bytes)
        return fail(TR_ERR_STRIDE, "%s: strides must be multiples of %d bytes", name, row_align_bytes);
    }
  }
  return TR_OK;
}
inline tr_status check_tensor(const char* name, const tr_tensor* t, bool allow_bf16, bool allow_f32, int row_align_bytes) {
  return check_typed(name, t, (allow_bf16 ? kBf16 : 0) | (allow_f32 ? kF32 : 0), row_align_bytes);
}

// A tensor the kernels write must not address one element through two index tuples (a zero or
// too small stride on a dimension larger than 1): rows are updated by different waves, so an
// overlapping view would race.  Sufficient test: ordered by stride, every dimension must step
// over the whole extent of the dimensions inside it.
inline tr_status check_written(const char* name, const tr_tensor* t) {
  if (extent_elems(t) == 0) return TR_OK;
  int64_t size[3] = {t->B, t->H, t->S}, stride[3] = {t->stride_b, t->stride_h, t->stride_s};
  for (int i = 0; i < 3; i++)
    for (int j = i + 1; j < 3; j++)
      if (stride[j] < stride[i]) {
        const int64_t a = size[i], b = stride[i];
        size[i] = size[j]; stride[i] = stride[j];
        size[j] = a; stride[j] = b;
      }
  int64_t inner = t->D;
  for (int i = 0; i < 3; i++) {
    if (size[i] <= 1) continue;
    if (stride[i] < inner) return fail(TR_ERR_STRIDE, "%s: a written tensor must not overlap itself (stride %lld < %lld elements inside it)", name, (long long)stride[i], (long long)inner);
    inner = stride[i] * (size[i] - 1) + inner;
  }
  return TR_OK;
}

}  // namespace tr
