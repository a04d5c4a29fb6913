// Whether two tensors share memory: rows of `width` bytes at up to three strides.  Exact where one of the two is nested (a row, or all rows of an inner axis, end before the next
// of the outer one begins, as in every view of a buffer by its axes), so that two slices of one buffer that lie between each other's rows pass.  No HIP in here: the CPU
// tests compile it as it is.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace basa {

struct RowSet {
  uint64_t at = 0, width = 0;               // of the first row; width 0: nothing
  int levels = 0;
  uint64_t n[3] = {}, stride[3] = {};       // outer axis first, none of one entry
};
// (A product beyond 2^62 stands for itself: no memory is that large.)
inline uint64_t reach_of(uint64_t n, uint64_t stride) {
  uint64_t r;
  return __builtin_mul_overflow(n, stride, &r) || r > (1ull << 62) ? 1ull << 62 : r;
}
// `strides` in bytes, axes in any order.  Axes whose rows meet or overlap are one longer row.
inline RowSet row_set(const void* at, uint64_t width, const uint64_t (&n)[3], const uint64_t (&strides)[3]) {
  RowSet s;
  s.at = reinterpret_cast<uintptr_t>(at);
  if (!at || !width || !n[0] || !n[1] || !n[2]) return s;
  s.width = width;
  bool used[3] = {n[0] == 1, n[1] == 1, n[2] == 1};
  for (;;) {                                // the axis with the smallest stride that is left
    int next = -1;
    for (int i = 0; i < 3; ++i)
      if (!used[i] && (next < 0 || strides[i] < strides[next])) next = i;
    if (next < 0) return s;
    used[next] = true;
    if (s.levels == 0 && strides[next] <= s.width) {
      s.width += reach_of(n[next] - 1, strides[next]);
      continue;
    }
    for (int i = s.levels++; i > 0; --i) { s.n[i] = s.n[i - 1]; s.stride[i] = s.stride[i - 1]; }
    s.n[0] = n[next]; s.stride[0] = strides[next];
  }
}
inline RowSet row_set(const void* at, uint64_t bytes) { return row_set(at, bytes, {1, 1, 1}, {0, 0, 0}); }
// Bytes from the first row's begin to the last one's end, of the levels from `level` on.
inline uint64_t span_of(const RowSet& s, int level = 0) {
  uint64_t span = s.width;
  for (int i = level; i < s.levels; ++i) span += reach_of(s.n[i] - 1, s.stride[i]);
  return span;
}
inline bool is_nested(const RowSet& s) {
  for (int i = 0; i < s.levels; ++i)
    if (span_of(s, i + 1) > s.stride[i]) return false;
  return true;
}
// Whether [x, x + bytes) meets a row of a nested set: the last row that begins in or before it does, or none.
inline bool meets(const RowSet& s, uint64_t x, uint64_t bytes) {
  const uint64_t last = x + bytes - 1;
  if (last < s.at) return false;
  uint64_t row = s.at;
  for (int i = 0; i < s.levels; ++i) {
    const uint64_t k = (last - row) / s.stride[i];
    row += (k < s.n[i] ? k : s.n[i] - 1) * s.stride[i];
  }
  return row + s.width > x;
}
inline uint64_t rows_in(const RowSet& s) {
  uint64_t r = 1;
  for (int i = 0; i < s.levels; ++i) r = reach_of(r, s.n[i]);
  return r;
}
inline bool overlap(const RowSet& a, const RowSet& b) {
  if (!a.width || !b.width || a.at >= b.at + span_of(b) || b.at >= a.at + span_of(a)) return false;
  const bool a_nested = is_nested(a), b_nested = is_nested(b);
  const uint64_t a_rows = rows_in(a), b_rows = rows_in(b);
  const bool walk_a = b_nested && (!a_nested || a_rows <= b_rows);
  // Both stand across their own rows, or the one that does is long to walk: taken for what they reach over.
  if ((!a_nested && !b_nested) || (walk_a ? a_rows : b_rows) > (1u << 24)) return true;
  const RowSet &walked = walk_a ? a : b, &other = walk_a ? b : a;
  uint64_t n[3] = {1, 1, 1}, stride[3] = {};
  for (int i = 0; i < walked.levels; ++i) { n[i] = walked.n[i]; stride[i] = walked.stride[i]; }
  for (uint64_t i = 0; i < n[0]; ++i)
    for (uint64_t j = 0; j < n[1]; ++j)
      for (uint64_t k = 0; k < n[2]; ++k)
        if (meets(other, walked.at + i * stride[0] + j * stride[1] + k * stride[2], walked.width)) return true;
  return false;
}

}  // namespace basa
