// Argument checks that the entry points of the handle-free operators share.  Host only.
#pragma once

#include "dw_ops.h"

namespace dw {
namespace {

#define DW_HIP(expr)                                          \
  do {                                                        \
    hipError_t e__ = (expr);                                  \
    if (e__ != hipSuccess) return note_hip_error(e__);        \
  } while (0)

inline bool is_type(int dtype) { return dtype == DW_F32 || dtype == DW_BF16; }
inline int64_t type_bytes(int dtype) { return dtype == DW_BF16 ? 2 : 4; }
inline bool aligned(const void* p, int64_t a) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(a - 1)) == 0; }

constexpr int64_t kMaxRows = 1ll << 31;                     // rows of a worker
constexpr int64_t kMaxStride = 1ll << 48;                   // elements: a byte offset stays in 64 bits for every worker

// rows of n at p that are only read
inline bool in_ok(const void* p, int64_t ld, int64_t stride, int64_t rows, int64_t n, int64_t bytes) {
  return aligned(p, bytes) && (rows <= 1 || ld >= n) && ld >= 0 && ld <= kMaxStride / (rows > 0 ? rows : 1) && stride >= 0 && stride <= kMaxStride;
}
// no two rows of k workers share an element (a worker's own do not, ld >= n): the workers lie one behind the other, or each row
// of a worker between two of worker 0's, or behind its last one
inline bool rows_apart(int64_t ld, int64_t stride, int k, int64_t rows, int64_t n) {
  if (k == 1 || rows == 0 || stride >= (rows - 1) * ld + n) return true;
  for (int w = 1; w < k; ++w) {                             // (what holds for the first rows of two workers holds for all w apart)
    const int64_t at = w * stride;
    const int64_t before = rows == 1 || at >= (rows - 1) * ld ? rows - 1 : at / ld;        // the last row of worker 0 that begins at or before
    if (at - before * ld < n || (before + 1 < rows && (before + 1) * ld - at < n)) return false;
  }
  return true;
}
// rows that are written: no two of them share an element
inline bool out_ok(const void* p, int64_t ld, int64_t stride, int k, int64_t rows, int64_t n, int64_t bytes) {
  return in_ok(p, ld, stride, rows, n, bytes) && rows_apart(ld, stride, k, rows, n);
}
inline bool params_ok(const float* p, int64_t stride) { return aligned(p, 4) && stride >= 0 && stride <= kMaxStride; }
inline bool grads_ok(const float* p, int64_t stride, int k, int64_t n) { return params_ok(p, stride) && (k == 1 || stride >= n); }

}  // namespace
}  // namespace dw
