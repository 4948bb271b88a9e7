// Rows held in 8 bits: e4m3 codes with one power of two for each row and 128 columns.
//
//   e = the least integer >= -126 with max |x| <= 448 2^e over the block's finite values,
//   code = x 2^-e rounded to e4m3 (nearest, ties to even), value = code 2^e
//
// 448 is e4m3's largest number, so no value is cut off.  The scale is a power of two and
// not max / 448: dividing and multiplying by it is exact, a code's value fits bf16, and
// it is the form in which the matrix instructions take scales.  It costs nothing in
// precision: e4m3 has exponents of its own, and a factor of at most two moves only what
// lies below 2^-14 of the largest value.  A scale byte s stands for 2^(s - 127).
// NaN and infinities become NaN codes and leave the block's other values alone.
#pragma once

#include "common.h"

namespace sscn {

constexpr int ROW8_BLOCK = 128;  // columns of a scale

__host__ __device__ inline int64_t row8_blocks(int64_t cols) { return (cols + ROW8_BLOCK - 1) / ROW8_BLOCK; }
// Bytes between rows: codes padded with zeros to 16 (whole vectors), scales to 4 (whole words).
__host__ __device__ inline int64_t row8_code_stride(int64_t cols) { return round_up(cols, 16); }
__host__ __device__ inline int64_t row8_scale_stride(int64_t cols) { return round_up(row8_blocks(cols), 4); }

// The scale byte of a block whose largest finite magnitude has bits `most`: 448 = 1.75 * 2^8, so
// the exponent is the magnitude's less 8, one more where its fraction passes 1.75.
__device__ inline uint32_t row8_scale(uint32_t most) {
  const int s = (int)((most + 0x1FFFFFu) >> 23) - 8;
  return (uint32_t)(s < 1 ? 1 : s);
}
__device__ inline float row8_pow2(uint32_t s) { return __uint_as_float(s << 23); }  // 2^(s - 127), s >= 1

__device__ inline bool is_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

typedef float row8_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 row8_bf16x2 __attribute__((ext_vector_type(2)));

// Four codes times a power of two, in float32 (exact).
__device__ inline void row8_values4(uint32_t w, float scale, float* f) {
  const row8_f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false);
  const row8_f32x2 hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
  f[0] = lo[0], f[1] = lo[1], f[2] = hi[0], f[3] = hi[1];
}

// A matrix [k][n] in 8 bits, one scale for each block of 128 x 128: the codes twice, along
// n and along k (each product reads them along its sum), rows padded with zeros to 128.
struct Weight8 {
  uint8_t* codes;     // [k][stride]
  uint8_t* codes_t;   // [n][stride_t]
  uint8_t* scales;    // [k blocks][scale_stride]
  uint8_t* scales_t;  // [n blocks][scale_stride_t]
  int64_t stride, stride_t;
  int32_t scale_stride, scale_stride_t;
};
__host__ __device__ inline Weight8 weight8_parts(uint8_t* base, int64_t k, int64_t n, int64_t* bytes = nullptr) {
  Weight8 w;
  w.stride = round_up(n, ROW8_BLOCK);
  w.stride_t = round_up(k, ROW8_BLOCK);
  w.scale_stride = (int32_t)row8_scale_stride(n);
  w.scale_stride_t = (int32_t)row8_scale_stride(k);
  int64_t at = 0;
  w.codes = base;
  at += k * w.stride;
  w.codes_t = base + at;
  at += n * w.stride_t;
  w.scales = base + at;
  at += round_up(row8_blocks(k) * w.scale_stride, 256);
  w.scales_t = base + at;
  at += round_up(row8_blocks(n) * w.scale_stride_t, 256);
  if (bytes) *bytes = at;
  return w;
}

}  // namespace sscn
