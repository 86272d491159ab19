// kv_strides.h -- what the host checks of arrays' strides.
#pragma once
#include <stdint.h>

namespace p2p {

// Rows of an array of 16-bit values, `dim` of them each at `at` + i * row + h * head (h < heads).
struct RowsAt {
  const void* at;
  int64_t row, head, heads;
};
// Whether rows of a and b (i < n of both) share a value; also said where their strides leave that open: they reach over
// the same memory with different distances from row to row, or with very many heads.
inline bool rows_meet(const RowsAt& a, const RowsAt& b, int64_t n, int64_t dim) {
  using wide = __int128;
  const wide apart = ((wide)(uintptr_t)b.at - (wide)(uintptr_t)a.at) / 2;
  const auto low = [n](const RowsAt& x) {
    return (x.row < 0 ? (wide)(n - 1) * x.row : 0) + (x.head < 0 ? (wide)(x.heads - 1) * x.head : 0);
  };
  const auto high = [n, dim](const RowsAt& x) {
    return (x.row > 0 ? (wide)(n - 1) * x.row : 0) + (x.head > 0 ? (wide)(x.heads - 1) * x.head : 0) + dim;
  };
  if (apart + low(b) >= high(a) || apart + high(b) <= low(a)) return false;
  if (n > 1 && a.row != b.row) return true;
  const wide row = n > 1 ? (a.row < 0 ? -(wide)a.row : a.row) : 0;
  if (row > 0 && a.head >= 0 && b.head >= 0) {  // parts of the same rows, as of queries, keys and values side by side
    wide d = apart % row;
    if (d < 0) d += row;
    if (d >= (wide)(a.heads - 1) * a.head + dim && d + (wide)(b.heads - 1) * b.head + dim <= row) return false;
  }
  // Whether rows that are d apart share a value, or others that are whole rows further apart or nearer.
  const auto meet = [n, dim, row](wide d) {
    if (row == 0) return d > -dim && d < dim;
    wide i = d / row;  // (rounded to zero: the nearest row is this one or the next on d's side, if there are so many)
    i = i >= n ? n - 1 : i <= -n ? 1 - n : i;
    for (int y = 0; y < 2; ++y, i += d < 0 ? -1 : 1) {
      const wide x = d - i * row;
      if (i > -n && i < n && x > -dim && x < dim) return true;
    }
    return false;
  };
  if (a.head == b.head) {
    for (int64_t h = 1 - a.heads; h < b.heads; ++h)
      if (meet(apart + (wide)h * a.head)) return true;
    return false;
  }
  if (a.heads * b.heads > 1 << 20) return true;
  for (int64_t x = 0; x < a.heads; ++x)
    for (int64_t y = 0; y < b.heads; ++y)
      if (meet(apart + (wide)y * b.head - (wide)x * a.head)) return true;
  return false;
}

}  // namespace p2p
