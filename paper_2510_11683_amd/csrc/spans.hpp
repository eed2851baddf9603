// Host-side checks of the arrays that an entry point takes.
#pragma once

#include <stdint.h>

namespace bgpo {

// The bytes [lo, hi) of an array (empty for NULL).
struct Span {
  uintptr_t lo, hi;
};

inline Span span(const void* p, int64_t bytes) {
  return p ? Span{(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes} : Span{0, 0};
}

// rows of `cols` elements of e bytes, ld elements apart
inline Span rows_span(const void* p, int64_t rows, int64_t ld, int64_t cols, int64_t e) {
  return span(p, ((rows - 1) * ld + cols) * e);
}

inline bool overlap(const Span& a, const Span& b) { return a.lo < b.hi && b.lo < a.hi; }

// whether an output shares bytes with an input or with another output
inline bool any_overlap(const Span* out, int n_out, const Span* in, int n_in) {
  for (int i = 0; i < n_out; ++i) {
    for (int j = 0; j < n_in; ++j)
      if (overlap(out[i], in[j])) return true;
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return true;
  }
  return false;
}

inline bool misaligned(const void* p, int64_t bytes) { return (uintptr_t)p & (uintptr_t)(bytes - 1); }

}  // namespace bgpo
