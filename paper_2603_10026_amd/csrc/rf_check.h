// Host-side checks of rf_tensor arguments shared by the C-ABI layer's files.
#pragma once
#include <stdint.h>

#include "../../include/rf.h"

namespace rf {
namespace check {

inline size_t esize(rf_dtype t) { return t == RF_BF16 ? 2 : t == RF_FP8_E4M3 ? 1 : 4; }  // f32, i32: 4
// `also`: one more dtype this argument may have (-1: none)
inline bool dtype_ok(rf_dtype t, int also) {
  return t == RF_F32 || t == RF_BF16 || (also >= 0 && (int)t == also);
}

// Structural checks common to every tensor argument.
// (integer and FP8 tensors are accepted only where an entry point asks for them)
inline rf_status check_tensor(const rf_tensor* t, int ndim_min, int ndim_max, int also = -1) {
  if (t == nullptr) return RF_ERR_INVALID_ARG;
  if (t->ndim < ndim_min || t->ndim > ndim_max) return RF_ERR_INVALID_ARG;
  if (!dtype_ok(t->dtype, also)) return RF_ERR_UNSUPPORTED;
  for (int i = 0; i < t->ndim; ++i) {
    if (t->shape[i] < 0 || t->stride[i] < 0) return RF_ERR_INVALID_ARG;
  }
  return RF_OK;
}

inline int64_t numel(const rf_tensor* t) {
  int64_t n = 1;
  for (int i = 0; i < t->ndim; ++i) n *= t->shape[i];
  return n;
}

inline bool same_shape(const rf_tensor* a, const rf_tensor* b) {
  if (a->ndim != b->ndim) return false;
  for (int i = 0; i < a->ndim; ++i)
    if (a->shape[i] != b->shape[i]) return false;
  return true;
}

inline bool is_contiguous(const rf_tensor* t) {
  int64_t expect = 1;
  for (int i = t->ndim - 1; i >= 0; --i) {
    if (t->shape[i] != 1 && t->stride[i] != expect) return false;
    expect *= t->shape[i];
  }
  return true;
}

// 16-byte alignment of the base pointer and of every outer stride.
inline bool aligned16(const rf_tensor* t) {
  if (reinterpret_cast<uintptr_t>(t->data) % 16 != 0) return false;
  for (int i = 0; i + 1 < t->ndim; ++i)
    if (t->shape[i] > 1 && (t->stride[i] * (int64_t)esize(t->dtype)) % 16 != 0) return false;
  return true;
}

// Leading dims collapse to `rows` rows with a single pitch?
inline bool collapse_rows(const rf_tensor* t, int64_t* rows, int64_t* pitch) {
  const int nd = t->ndim;
  int64_t r = 1;
  for (int i = 0; i + 1 < nd; ++i) r *= t->shape[i];
  *rows = r;
  if (nd == 1) { *pitch = t->shape[0]; return true; }
  *pitch = t->stride[nd - 2];
  for (int i = nd - 3; i >= 0; --i) {
    if (t->shape[i] == 1) continue;
    if (t->stride[i] != t->stride[i + 1] * t->shape[i + 1]) return false;
  }
  if (r > 1 && *pitch < t->shape[nd - 1]) return false;
  return true;
}

}  // namespace check
}  // namespace rf
