// Host-side checks of tensor descriptors, shared by the entry points.
#pragma once

#include <cstdint>

#include "dlm_internal.h"
#include "dlmrefine.h"

namespace dlm {

inline int64_t elem_size(int dtype) {
  switch (dtype) {
    case DLM_BF16: return 2;
    case DLM_F32: return 4;
    case DLM_I32: return 4;
    case DLM_U8: return 1;
    default: return 0;
  }
}

inline int64_t numel(const dlm_tensor* t) {
  for (int i = 0; i < t->ndim; ++i)
    if (t->shape[i] == 0) return 0;
  int64_t n = 1;
  for (int i = 0; i < t->ndim; ++i) n *= t->shape[i];
  return n;
}

// Checks pointer, dtype, rank, non-negative extents and a contiguous innermost
// dimension. `name` appears in the error message. most: the largest extent; the number of
// elements fits 62 bits in any case.
inline int check_tensor(const dlm_tensor* t, const char* name, int dtype_mask, int ndim_lo, int ndim_hi,
                        int64_t most = 0x7FFFFFFF) {
  if (!t) return fail(DLM_ERR_NULL, "%s: descriptor is NULL", name);
  if (elem_size(t->dtype) == 0 || !((1 << t->dtype) & dtype_mask))
    return fail(DLM_ERR_DTYPE, "%s: unsupported dtype %d", name, t->dtype);
  if (t->ndim < ndim_lo || t->ndim > ndim_hi)
    return fail(DLM_ERR_SHAPE, "%s: rank %d not in [%d, %d]", name, t->ndim, ndim_lo, ndim_hi);
  for (int i = 0; i < t->ndim; ++i) {
    if (t->shape[i] < 0) return fail(DLM_ERR_SHAPE, "%s: negative extent", name);
    if (t->shape[i] > most) return fail(DLM_ERR_SHAPE, "%s: extent too large", name);
  }
  double elements = 1;
  for (int i = 0; i < t->ndim; ++i) elements *= static_cast<double>(t->shape[i]);
  if (elements > 0x1p62) return fail(DLM_ERR_SHAPE, "%s: too many elements", name);
  if (numel(t) > 0) {
    if (!t->data) return fail(DLM_ERR_NULL, "%s: data pointer is NULL", name);
    if (t->shape[t->ndim - 1] > 1 && t->stride[t->ndim - 1] != 1)
      return fail(DLM_ERR_STRIDE, "%s: innermost dimension must be contiguous", name);
    for (int i = 0; i < t->ndim; ++i)
      if (t->stride[i] < 0) return fail(DLM_ERR_STRIDE, "%s: negative stride", name);
    if (reinterpret_cast<uintptr_t>(t->data) % static_cast<uintptr_t>(elem_size(t->dtype)) != 0)
      return fail(DLM_ERR_ALIGN, "%s: data pointer not aligned to its element size", name);
  }
  return DLM_OK;
}

inline bool is_dense(const dlm_tensor* t) {
  if (numel(t) == 0) return true;
  int64_t expect = 1;
  for (int i = t->ndim - 1; i >= 0; --i) {
    if (t->shape[i] > 1 && t->stride[i] != expect) return false;
    expect *= t->shape[i];
  }
  return true;
}

// Byte range [lo, hi) touched by a strided tensor.
inline void byte_span(const dlm_tensor* t, uintptr_t* lo, uintptr_t* hi) {
  int64_t last = 0;
  for (int i = 0; i < t->ndim; ++i)
    if (t->shape[i] > 0) last += (t->shape[i] - 1) * t->stride[i];
  *lo = reinterpret_cast<uintptr_t>(t->data);
  *hi = *lo + static_cast<uintptr_t>((last + 1) * elem_size(t->dtype));
}

inline bool overlaps(const dlm_tensor* a, const dlm_tensor* b) {
  if (numel(a) == 0 || numel(b) == 0) return false;
  uintptr_t alo, ahi, blo, bhi;
  byte_span(a, &alo, &ahi);
  byte_span(b, &blo, &bhi);
  return alo < bhi && blo < ahi;
}

inline bool same_view(const dlm_tensor* a, const dlm_tensor* b) {
  if (a->data != b->data || a->ndim != b->ndim || a->dtype != b->dtype) return false;
  for (int i = 0; i < a->ndim; ++i)
    if (a->shape[i] != b->shape[i] || (a->shape[i] > 1 && a->stride[i] != b->stride[i])) return false;
  return true;
}

constexpr int kMaskBF16F32 = (1 << DLM_BF16) | (1 << DLM_F32);

}  // namespace dlm
