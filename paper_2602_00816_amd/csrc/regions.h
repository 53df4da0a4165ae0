// Overlap of caller-owned operands, for the argument checks of the calls that take
// them one by one (host code).
#pragma once
#include <cstddef>
#include <cstdint>

namespace fdh {

// rows of `width` bytes, `ld` bytes apart
struct Region {
  const char* p;
  int64_t rows, ld, width;
};
inline Region flat(const void* p, int64_t bytes) { return {(const char*)p, 1, bytes, bytes}; }

// whether a byte of one may lie in the other: regions of the same row stride are
// told apart by their columns (two slices of one wide buffer do not overlap)
inline bool overlap(const Region& a, const Region& b) {
  if (!a.p || !b.p || a.rows == 0 || b.rows == 0 || a.width == 0 || b.width == 0) return false;
  const Region &lo = a.p <= b.p ? a : b, &hi = a.p <= b.p ? b : a;
  const int64_t gap = hi.p - lo.p;
  if (gap >= (lo.rows - 1) * lo.ld + lo.width) return false;
  if (lo.ld != hi.ld) return true;
  const int64_t c = gap % lo.ld;
  return !(c >= lo.width && lo.ld - c >= hi.width);
}

// whether one of the written regions w overlaps another of them or a region r that is read
inline bool any_overlap(const Region* w, int nw, const Region* r, int nr) {
  for (int i = 0; i < nw; ++i) {
    for (int j = i + 1; j < nw; ++j)
      if (overlap(w[i], w[j])) return true;
    for (int j = 0; j < nr; ++j)
      if (overlap(w[i], r[j])) return true;
  }
  return false;
}

// a [rows][ld] operand of `size`-byte elements: 16-byte accesses and row offsets in 64 bits
inline bool bad_rows(const void* p, int64_t ld, int64_t cols, int size) {
  return !p || (uintptr_t)p % 16 || ld < cols || ld > ((int64_t)1 << 31) || ld * size % 16;
}

}  // namespace fdh
