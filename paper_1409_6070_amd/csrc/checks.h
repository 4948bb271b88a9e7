// Checks of arguments that the calls on plain arrays share.
#pragma once

#include <algorithm>
#include <cstdint>
#include <memory>
#include <new>

#include "sscn.h"
#include "common.h"
#include "spans.h"

namespace sscn {

inline bool known_dtype(int32_t dtype) { return dtype == SSCN_F32 || dtype == SSCN_BF16; }

inline size_t aligned256(size_t n) { return (n + 255) / 256 * 256; }

inline sscn_status of_hip(hipError_t e) { return e == hipSuccess ? SSCN_OK : SSCN_ERR_HIP; }

// Elements from an array's first to its last, at most: their bytes fit 63 bits.
constexpr int64_t MAX_SPAN = (int64_t)1 << 60;

// rows x cols elements with `stride` elements between rows (both below 2^32: no overflow here)
inline bool rows_ok(int64_t rows, int64_t cols, int64_t stride) {
  return rows >= 0 && rows <= SSCN_MAX_ROWS && stride >= cols && stride <= ((int64_t)1 << 31) &&
         (rows <= 1 || (rows - 1) * stride + cols <= MAX_SPAN);
}

inline bool bad_workspace(const void* ws, size_t have, size_t need) {
  return need > 0 && (!ws || have < need || (uintptr_t)ws % 256 != 0);
}

// Refuses arrays of which one that is written overlaps another: fill(list) sets at most
// `most` of them and returns how many.
template <class Fill>
sscn_status apart(int64_t most, Fill&& fill) {
  Span few[64];
  std::unique_ptr<Span[]> many;
  Span* list = few;
  if (most > 64) {
    many.reset(new (std::nothrow) Span[most]);
    if (!many) return SSCN_ERR_INVALID_ARGUMENT;
    list = many.get();
  }
  return outputs_overlap(list, fill(list)) ? SSCN_ERR_INVALID_ARGUMENT : SSCN_OK;
}

}  // namespace sscn
