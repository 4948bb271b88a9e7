// Sums over lanes of a wave.
#pragma once

#include "common.h"

namespace sscn {

template <int CTRL>
__device__ inline float add_dpp(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

// Sum over aligned groups of G lanes, in every lane of the group (each level
// adds the two halves in the same order in both, so all lanes agree bit for bit).
template <int G>
__device__ inline float group_sum(float v) {
  static_assert(G == 8 || G == 16 || G == 32 || G == 64, "lanes of a row");
  v = add_dpp<0xB1>(v);   // quad_perm 1,0,3,2
  v = add_dpp<0x4E>(v);   // quad_perm 2,3,0,1
  v = add_dpp<0x141>(v);  // row_half_mirror: the other quad of eight
  if constexpr (G >= 16) v = add_dpp<0x140>(v);  // row_mirror: the other eight of sixteen
  if constexpr (G >= 32) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
  if constexpr (G >= 64) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
  return v;
}

}  // namespace sscn
