// overlap.cuh -- whether strided tensors share elements (host side, internal header).
#pragma once

#include <stdint.h>

#include <algorithm>

namespace occam {

// A tensor's values as intervals of `width` elements at base + r row + h head.
struct Extent {
  __int128 base, row, head, rows, heads, width;  // base in elements
  __int128 end() const { return base + (rows - 1) * row + (heads - 1) * head + width; }
};
inline Extent extent(const void* at, int64_t rows, int64_t row, int64_t heads, int64_t head, int64_t dim, int64_t es) {
  Extent e{(__int128)(reinterpret_cast<uintptr_t>(at) / es), row, head, rows, heads, dim};
  if (e.rows == 1 || e.row == 0) e.rows = 1, e.row = 0;      // (a row read again is one row)
  if (e.heads == 1 || e.head == 0) e.heads = 1, e.head = 0;
  if (e.head == e.width) e.width *= e.heads, e.heads = 1, e.head = 0;  // heads side by side are one interval
  return e;
}
// Whether c + n pitch lies in lo .. hi for some n in first .. last (pitch >= 0).
inline bool reaches(__int128 c, __int128 pitch, __int128 first, __int128 last, __int128 lo, __int128 hi) {
  if (pitch == 0) return lo <= c && c <= hi;
  auto floor_div = [](__int128 a, __int128 b) { return a >= 0 ? a / b : -((-a + b - 1) / b); };
  const __int128 n = std::max(first, -floor_div(c - lo, pitch));  // the least n with c + n pitch >= lo
  return n <= last && c + n * pitch <= hi;
}
// Whether two tensors have an element in common. (Exact, but for tensors that lie within each other with
// rows of different strides, or more than 2^20 pairs of heads with different strides: true.)
inline bool meet(const Extent& a, const Extent& b) {
  if (a.end() <= b.base || b.end() <= a.base) return false;
  if (a.rows > 1 && b.rows > 1 && a.row != b.row) return true;
  const __int128 pitch = a.rows > 1 ? a.row : b.row, at = a.base - b.base;
  auto rows_meet = [&](__int128 c) { return reaches(c, pitch, 1 - b.rows, a.rows - 1, 1 - a.width, b.width - 1); };
  if (a.heads == 1 || b.heads == 1 || a.head == b.head) {
    const __int128 head = a.heads > 1 ? a.head : b.head;
    for (__int128 h = 1 - b.heads; h < a.heads; ++h)
      if (rows_meet(at + h * head)) return true;
    return false;
  }
  if (a.heads * b.heads > (1 << 20)) return true;
  for (__int128 h = 0; h < a.heads; ++h)
    for (__int128 k = 0; k < b.heads; ++k)
      if (rows_meet(at + h * a.head - k * b.head)) return true;
  return false;
}
// Whether two of a tensor's own (row, head) intervals have an element in common.
inline bool meets_itself(const Extent& a) {
  if (a.row >= (a.heads - 1) * a.head + a.width || a.rows == 1) return a.heads > 1 && a.head < a.width;
  if (a.heads == 1) return true;  // (rows closer than a row is wide)
  if (a.head >= (a.rows - 1) * a.row + a.width) return a.row < a.width;
  for (__int128 h = 0; h < a.heads; ++h)  // h = 0: rows 1 .. apart
    if (reaches(h * a.head, a.row, h ? 1 - a.rows : 1, a.rows - 1, 1 - a.width, a.width - 1)) return true;
  return false;
}

}  // namespace occam
