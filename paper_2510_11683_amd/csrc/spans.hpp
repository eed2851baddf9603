// Host-side checks of the arrays that an entry point takes.
#pragma once

#include <stdint.h>

namespace bgpo {

// rows x cols elements of e bytes, row starts ld elements apart; p NULL: none.
struct Array {
  const void* p;
  int64_t rows, ld, cols, e;
  uintptr_t begin() const { return (uintptr_t)p; }
  uintptr_t end() const { return begin() + (uintptr_t)(((rows - 1) * ld + cols) * e); }
};

inline Array vec(const void* p, int64_t n, int64_t e) { return Array{p, 1, 0, n, e}; }

// Whether two arrays share bytes.  Rows of one may lie between rows of the
// other where the strides are equal.
inline bool overlap(const Array& a, const Array& b) {
  if (!a.p || !b.p || a.end() <= b.begin() || b.end() <= a.begin()) return false;
  const uintptr_t pa = (uintptr_t)(a.ld * a.e), pb = (uintptr_t)(b.ld * b.e);
  const uintptr_t pitch = a.rows > 1 ? pa : pb;
  if ((a.rows <= 1 && b.rows <= 1) || (a.rows > 1 && b.rows > 1 && pa != pb)) return true;
  const uintptr_t at = b.begin() >= a.begin() ? (b.begin() - a.begin()) % pitch
                                              : (pitch - (a.begin() - b.begin()) % pitch) % pitch;
  return !(at >= (uintptr_t)(a.cols * a.e) && at + (uintptr_t)(b.cols * b.e) <= pitch);
}

// whether an output shares bytes with an input or with another output
template <int NO, int NI>
inline bool any_overlap(const Array (&out)[NO], const Array (&in)[NI]) {
  for (int i = 0; i < NO; ++i) {
    for (int j = 0; j < NI; ++j)
      if (overlap(out[i], in[j])) return true;
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return true;
  }
  return false;
}

// a stride between rows that is too small, or past any memory (any value will
// do where there is one row or no array)
inline bool bad_stride(const void* p, int64_t ld, int64_t rows, int64_t cols) {
  return p && rows > 1 && (ld < cols || ld > (int64_t(1) << 56) / rows);
}

inline bool misaligned(const void* p, int64_t bytes) { return (uintptr_t)p & (uintptr_t)(bytes - 1); }

}  // namespace bgpo
