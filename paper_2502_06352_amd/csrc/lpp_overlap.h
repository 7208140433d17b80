// Whether what a call writes lies in what it reads.  Host code alone: tests/test_overlap.py tries it.
#ifndef LPP_OVERLAP_H_
#define LPP_OVERLAP_H_

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

// `na` bytes at a and `nb` bytes at b (null: nothing is there)
inline bool ranges_meet(const void* a, uint64_t na, const void* b, uint64_t nb) {
  const uint64_t x = (uint64_t)(uintptr_t)a, y = (uint64_t)(uintptr_t)b;
  return a && b && na && nb && x < y + nb && y < x + na;
}

// B x M x heads rows of `width` bytes, strides in bytes and none negative, and `n` bytes at `out`.  Exact: the rows may have what is written
// between them.  Tensors of their own are told apart by where they begin and end.
inline bool rows_meet(const void* data, int64_t item, int64_t row, int64_t head, int64_t B, int64_t M, int64_t heads, int64_t width, const void* out,
                      int64_t n) {
  const int64_t first = (int64_t)(uintptr_t)data, lo = (int64_t)(uintptr_t)out, hi = lo + n;
  const int64_t end = first + (B - 1) * item + (M - 1) * row + (heads - 1) * head + width;
  if (first >= hi || end <= lo) return false;
  if (item == M * row) { M *= B; B = 1; }
  if (row == 0) M = 1;
  for (int64_t b = 0; b < (item == 0 ? 1 : B); ++b)
    for (int64_t h = 0; h < (head == 0 ? 1 : heads); ++h) {
      const int64_t at = first + b * item + h * head;                // row i begins at at + i row
      const int64_t i = lo - width < at || row == 0 ? 0 : (lo - width - at) / row + 1;        // the first that ends behind lo
      if (i < M && at + i * row < hi && at + i * row + width > lo) return true;
    }
  return false;
}

#endif  // LPP_OVERLAP_H_
