// overlap.h -- whether two strided pieces of memory share a byte (host only, no CUDA).
//
// Outputs and inputs may be columns of the same wider buffer, side by side, so
// that comparing addresses, or first and last bytes, is not enough.
#pragma once

#include <cstdint>
#include <cstdio>
#include <initializer_list>

namespace bds {

struct Span {  // `rows` pieces of `row` bytes, `ld` bytes apart (row <= ld); at null: none
  const char* name;
  const void* at;
  int64_t rows, row, ld;
};

inline Span dense_span(const char* name, const void* at, int64_t bytes) { return Span{name, at, 1, bytes, bytes}; }

// Whether bytes lo .. lo + n - 1 hold one of b's.
inline bool overlaps_row(int64_t lo, int64_t n, const Span& b) {
  const int64_t from = lo - (int64_t)(uintptr_t)b.at;  // relative to b's first byte
  // b's first piece that ends behind it
  const int64_t j = from < b.row ? 0 : (from - b.row) / b.ld + 1;
  return j < b.rows && j * b.ld < from + n;
}

inline bool overlap(Span a, Span b) {
  if (a.at == nullptr || b.at == nullptr || a.rows <= 0 || b.rows <= 0 || a.row <= 0 || b.row <= 0) return false;
  for (Span* s : {&a, &b})  // pieces without gaps are one
    if (s->rows == 1 || s->row == s->ld) *s = dense_span(s->name, s->at, s->row * s->rows);
  const int64_t a0 = (int64_t)(uintptr_t)a.at, b0 = (int64_t)(uintptr_t)b.at;
  if (a0 + (a.rows - 1) * a.ld + a.row <= b0 || b0 + (b.rows - 1) * b.ld + b.row <= a0) return false;
  // of the same stride, pieces i and i + k share what pieces i - 1 and i - 1 + k do: the first of either decides
  if (a.rows > 1 && a.ld == b.ld) return overlaps_row(a0, a.row, b) || overlaps_row(b0, b.row, a);
  const Span &few = a.rows < b.rows ? a : b, &many = a.rows < b.rows ? b : a;
  for (int64_t i = 0; i < few.rows; ++i)
    if (overlaps_row((int64_t)(uintptr_t)few.at + i * few.ld, few.row, many)) return true;
  return false;
}

// Says in `msg` which of what a call reads shares memory with what it writes, if any does.
inline bool any_overlap(std::initializer_list<Span> reads, std::initializer_list<Span> writes, char* msg, size_t size) {
  for (const Span& w : writes)
    for (const Span& r : reads)
      if (overlap(r, w)) {
        snprintf(msg, size, "%s overlaps %s, which the call writes", r.name, w.name);
        return true;
      }
  return false;
}

}  // namespace bds
