// The bytes of a matrix or vector argument, and whether two of them meet.
#pragma once

#include <stdint.h>

#include <initializer_list>

namespace xema {

// `rows` runs of `width` bytes, `pitch` bytes apart (one run: a vector or a
// contiguous matrix); no bytes where p is null.
struct Span {
  const void* p;
  int64_t width, rows = 1, pitch = 0;
};

inline Span span_rows(const void* p, int64_t width, int64_t rows, int64_t pitch) {
  return width == pitch ? Span{p, width * rows} : Span{p, width, rows, pitch};
}

// Exact where both have one pitch or one of them is a single run, so that two
// column ranges of one buffer are apart.  Rows of unlike pitch are taken for
// the whole of what they span.
inline bool overlaps(Span a, Span b) {
  if (!a.p || !b.p || a.width <= 0 || b.width <= 0 || a.rows <= 0 || b.rows <= 0) return false;
  if (a.rows > 1 && b.rows > 1 && a.pitch != b.pitch) {
    a = {a.p, (a.rows - 1) * a.pitch + a.width};
    b = {b.p, (b.rows - 1) * b.pitch + b.width};
  }
  // row i of a meets row j of b where b - width(a) < (i - j) pitch < b + width(b), from a's start
  const int64_t at = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p);
  const int64_t pitch = a.rows > 1 ? a.pitch : b.rows > 1 ? b.pitch : 1;
  auto floor_div = [](int64_t n, int64_t d) { return n / d - (n % d < 0); };
  int64_t least = floor_div(at - a.width, pitch) + 1, most = -floor_div(-(at + b.width), pitch) - 1;
  if (least < -(b.rows - 1)) least = -(b.rows - 1);
  if (most > a.rows - 1) most = a.rows - 1;
  return least <= most;
}

inline bool any_overlap(const Span& out, std::initializer_list<Span> others) {
  for (const Span& o : others)
    if (overlaps(out, o)) return true;
  return false;
}

}  // namespace xema
