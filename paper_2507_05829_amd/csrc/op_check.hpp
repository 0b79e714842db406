// What the operators beside the row-wise products check of their arguments, on the host, before anything is enqueued.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "lop.h"
#include "plan_state.hpp"

namespace lop {

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
// A tensor that 16-byte vectors are moved through: non-null, on a 16-byte boundary, as is whatever a stride leads to (`used`: the
// extent is more than 1). Strides are not negative: the kernels' offsets are not.
inline bool whole_vectors(long long stride, size_t element, bool used) {
  return !used || (stride >= 0 && (size_t)stride * element % 16 == 0);
}
// Rows (or heads) of an output of `extent` elements do not overlap.
inline bool apart(long long stride, long long extent, long long count) { return count <= 1 || stride >= extent; }
// The same where the rows have heads (or any two orders of pieces of `extent` elements): no two pieces share an element. One order within the other's stride is
// the usual case; else row i against head j: the nearest rows to j heads' way, as far as there are that many.
inline bool apart(long long extent, long long stride, long long count, long long other_stride, long long other_count) {
  if (count <= 1 || other_count <= 1) return apart(stride, extent, count) && apart(other_stride, extent, other_count);
  if (stride > other_stride) return apart(extent, other_stride, other_count, stride, count);
  if (stride < extent) return false;
  if ((other_stride - extent) / stride >= count - 1) return true;
  for (long long j = 1; j < other_count; ++j) {
    const __int128 at = (__int128)j * other_stride, i = at / stride, past = at % stride;
    if (i > count - 1) break;
    if (past < extent || (i < count - 1 && stride - past < extent)) return false;
  }
  return true;
}
inline size_t dtype_bytes(int dtype) { return dtype == LOP_BF16 ? 2 : 4; }
inline bool known_dtype(int dtype) { return dtype == LOP_F32 || dtype == LOP_BF16; }
// LOP_OK, or what a band that is no interval of `total` rows is
inline int check_band(lop_rows_t r, long long total) { return r.lo < 0 || r.hi < r.lo || r.hi > total ? LOP_ERR_BAND_RANGE : LOP_OK; }
// Workgroups of one dimension that a launch takes: fewer than 2^32 threads (exclusive).
constexpr long long launch_blocks(int threads) { return 0xffffffffLL / threads; }
constexpr long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

}  // namespace lop
