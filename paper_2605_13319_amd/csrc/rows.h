// What callers' rows look like (host code).
#pragma once

#include <stdint.h>

#include <utility>

namespace pipesd {

// Whether a row of a and a row of b share bytes: `rows` of `width` bytes each, strides of at least that.
inline bool rows_overlap(const void* a, int64_t a_stride, const void* b, int64_t b_stride, int64_t rows, int64_t width) {
  if ((uintptr_t)a > (uintptr_t)b) std::swap(a, b), std::swap(a_stride, b_stride);
  int64_t at = (int64_t)((uintptr_t)b - (uintptr_t)a);  // of b's first row, from a's
  if (at >= (rows - 1) * a_stride + width) return false;
  if (a_stride == b_stride) {  // (columns of one matrix) b's rows lie between the same two rows of a each, or behind the last
    const int64_t before = at / a_stride;
    return at % a_stride < width || (before + 1 < rows && a_stride - at % a_stride < width);
  }
  for (int64_t i = 0, j = 0; i < rows && j < rows;) {
    if (at >= width) ++i, at -= a_stride;
    else if (at <= -width) ++j, at += b_stride;
    else return true;
  }
  return false;
}

}  // namespace pipesd
