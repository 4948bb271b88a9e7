// Whether the arrays of one call overlap where one of them is written.  Plain host code,
// so a host program can run the same text.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace sscn {

// `rows` runs of `len` bytes, `step` bytes apart (rows >= 1, step >= len where rows > 1).
struct Span {
  uint64_t at;
  int64_t rows, len, step;
  bool out;          // written
  int32_t in_place;  // arrays of one number >= 0 may be the same array, both ends and stride
};

inline Span span(const void* at, int64_t rows, int64_t len, int64_t step, bool out, int32_t in_place = -1) {
  return Span{(uint64_t)(uintptr_t)at, rows, len, rows > 1 ? step : 0, out, in_place};
}

inline uint64_t span_end(const Span& s) { return s.at + (uint64_t)((s.rows - 1) * s.step + s.len); }

// Whether a byte belongs to both.  Exact where the strides agree or one of them has a
// single row; arrays of different strides count as overlapping where their ranges do.
inline bool spans_meet(const Span& a, const Span& b) {
  if (a.at >= span_end(b) || b.at >= span_end(a)) return false;
  const int64_t step = a.rows > 1 ? a.step : b.step;
  if ((a.rows > 1 && b.rows > 1 && a.step != b.step) || step == 0) return true;
  // row r of a and q of b meet where k step - b.len < d < k step + a.len with k = r - q
  const int64_t d = (int64_t)(b.at - a.at);
  const auto floor_div = [&](int64_t x) { return x / step - (x % step < 0 ? 1 : 0); };
  const int64_t least = floor_div(d - a.len) + 1, most = -floor_div(-(d + b.len)) - 1;
  return std::max(least, 1 - b.rows) <= std::min(most, a.rows - 1);
}

// Whether an array that is written overlaps another one.  Sorts s.
inline bool outputs_overlap(Span* s, int64_t n) {
  std::sort(s, s + n, [](const Span& a, const Span& b) { return a.at < b.at; });
  for (int64_t i = 0; i < n; ++i)
    for (int64_t j = i + 1; j < n && s[j].at < span_end(s[i]); ++j) {
      if (!s[i].out && !s[j].out) continue;
      if (s[i].in_place >= 0 && s[i].in_place == s[j].in_place && s[i].at == s[j].at && s[i].rows == s[j].rows &&
          s[i].len == s[j].len && s[i].step == s[j].step)
        continue;
      if (spans_meet(s[i], s[j])) return true;
    }
  return false;
}

}  // namespace sscn
