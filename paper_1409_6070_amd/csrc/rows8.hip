// Rows and matrices to 8 bits and back (the format: rows8.h).

#include "common.h"
#include "kernels.h"
#include "rows8.h"

#include <algorithm>

namespace sscn {

namespace {

// Eight consecutive elements from an address aligned to one, of which the first n exist.
template <typename T>
struct Run8 {
  T e[8];
};
template <typename T>
__device__ inline Run8<T> load_run(const T* p, int n) {
  Run8<T> r;
  if (n >= 8) {
    __builtin_memcpy(&r, p, sizeof(r));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) r.e[e] = e < n ? p[e] : Elem<T>::from_f32(0.f);
  }
  return r;
}

// The bits of a run's largest magnitude, at least 0x7f800000 where one is not finite.  As integers:
// a maximum of floats loses what it has at a signalling NaN.
__device__ inline uint32_t largest(const Run8<float>& r) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(r.e[e]) & 0x7fffffffu);
  return m;
}
__device__ inline uint32_t largest(const Run8<__bf16>& r) {
  typedef uint16_t U16x2 __attribute__((ext_vector_type(2)));
  uint32_t w[4];
  __builtin_memcpy(w, &r, sizeof(r));
  U16x2 m = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    m = __builtin_elementwise_max(m, __builtin_bit_cast(U16x2, w[i] & 0x7fff7fffu));
  return (uint32_t)max(m[0], m[1]) << 16;
}
// ... of its finite values.
template <typename T>
__device__ inline uint32_t largest_finite(const Run8<T>& r) {
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float f = fabsf(Elem<T>::to_f32(r.e[e]));
    m = fmaxf(m, is_finite(f) ? f : 0.f);
  }
  return __float_as_uint(m);
}

typedef int16_t I16x2 __attribute__((ext_vector_type(2)));

// Codes under scale byte s: values that are NaN become NaN.
__device__ inline uint2 codes_of(const Run8<float>& r, uint32_t s) {
  const float scale = row8_pow2(s);
  I16x2 w[2] = {{0, 0}, {0, 0}};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w[i], r.e[4 * i], r.e[4 * i + 1], scale, false);
    w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w[i], r.e[4 * i + 2], r.e[4 * i + 3], scale, true);
  }
  return uint2{__builtin_bit_cast(uint32_t, w[0]), __builtin_bit_cast(uint32_t, w[1])};
}
__device__ inline uint2 codes_of(const Run8<__bf16>& r, uint32_t s) {
  const float scale = row8_pow2(s);
  row8_bf16x2 x[4];
  __builtin_memcpy(x, &r, sizeof(r));
  I16x2 w[2] = {{0, 0}, {0, 0}};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w[i], x[2 * i], scale, false);
    w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w[i], x[2 * i + 1], scale, true);
  }
  return uint2{__builtin_bit_cast(uint32_t, w[0]), __builtin_bit_cast(uint32_t, w[1])};
}
// ... and infinities too.
template <typename T>
__device__ inline Run8<T> without_infinities(Run8<T> r) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (!is_finite(Elem<T>::to_f32(r.e[e]))) r.e[e] = Elem<T>::from_f32(__uint_as_float(0x7fc00000u));
  return r;
}
constexpr uint32_t NOT_FINITE = 0x7f800000u;

template <int CTRL>
__device__ inline uint32_t max_dpp(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true));
}
// Largest over aligned groups of 16 lanes, in all of them.
__device__ inline uint32_t max16(uint32_t v) {
  v = max_dpp<0xB1>(v);   // quad_perm 1,0,3,2
  v = max_dpp<0x4E>(v);   // quad_perm 2,3,0,1
  v = max_dpp<0x141>(v);  // row_half_mirror
  return max_dpp<0x140>(v);  // row_mirror
}

// A workgroup takes R rows at a time, 16 lanes a block of 128 columns, eight columns a lane;
// PER blocks a lane group are in flight together.
constexpr int PER = 4, GROUPS = 16, ITEMS = PER * GROUPS;
constexpr int NO_ITEM = -(1 << 30);

__device__ inline int div_by(int i, int nb, float rcp) {
  int q = (int)((float)i * rcp);
  q += (q + 1) * nb <= i ? 1 : 0;
  q -= q * nb > i ? 1 : 0;
  return q;
}

// Bound by memory: 200001 x 1000 bf16 (606 MB) 121 to 126 us, 4.8 to 5.0 TB/s; by its launch where
// rows are few: 100 x 300 f32 4.3.
template <typename T>
__global__ void __launch_bounds__(256) k_rows8_store(Rows8Args a, int R, int64_t tiles) {
  const int nb = (int)row8_blocks(a.cols), lane = threadIdx.x & 15, group = threadIdx.x >> 4;
  const int64_t cs = row8_code_stride(a.cols), ss = row8_scale_stride(a.cols);
  const float rcp = 1.f / (float)nb;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t row0 = tile * R;
    const int n = (int)min((int64_t)R, a.rows - row0) * nb;
    for (int i0 = 0; i0 < n; i0 += ITEMS) {
      Run8<T> x[PER];
      int row[PER], blk[PER], live[PER];
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        const int i = i0 + p * GROUPS + group;
        row[p] = nb > ITEMS ? 0 : div_by(i, nb, rcp);  // (more blocks than a tile's items: a row at a time)
        blk[p] = i - row[p] * nb;
        const int c = blk[p] * ROW8_BLOCK + lane * 8;
        live[p] = i < n ? a.cols - c : NO_ITEM;  // this lane's elements: more than eight, some, or none
        x[p] = load_run<T>((const T*)a.x + (row0 + row[p]) * a.x_stride + c, live[p]);
      }
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        uint32_t most = max16(largest(x[p]));
        if (most >= NOT_FINITE) {  // (the block's sixteen lanes together)
          most = max16(largest_finite(x[p]));
          x[p] = without_infinities(x[p]);
        }
        const uint32_t s = row8_scale(most);
        if (live[p] == NO_ITEM) continue;
        const uint2 w = codes_of(x[p], s);
        const int c = blk[p] * ROW8_BLOCK + lane * 8;
        if (c < cs) *(uint2*)(a.codes + (row0 + row[p]) * cs + c) = w;
        uint8_t* sc = a.scales + (row0 + row[p]) * ss + blk[p];
        if (lane == 0) *sc = (uint8_t)s;
        if (blk[p] == nb - 1 && lane > 0 && lane < ss - blk[p]) sc[lane] = 0;
      }
    }
  }
}

// Bound by memory: 200001 x 1000 bf16 95 to 108 us, 5.6 to 6.4 TB/s with the codes partly from the
// last-level cache; 100 x 300 f32 4.1.
template <typename T>
__global__ void __launch_bounds__(256) k_rows8_load(Rows8Args a, int R, int64_t tiles) {
  constexpr int V = Elem<T>::VE, N = 8 / V;  // a lane's columns: N runs of 16 bytes, 16 V columns apart
  const int nb = (int)row8_blocks(a.cols), lane = threadIdx.x & 15, group = threadIdx.x >> 4;
  const int64_t cs = row8_code_stride(a.cols), ss = row8_scale_stride(a.cols);
  const float rcp = 1.f / (float)nb;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t row0 = tile * R;
    const int n = (int)min((int64_t)R, a.rows - row0) * nb;
    for (int i0 = 0; i0 < n; i0 += ITEMS) {
      uint32_t w[PER][N][V / 4], s[PER];
      int row[PER], col[PER], live[PER];
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        const int i = i0 + p * GROUPS + group;
        row[p] = nb > ITEMS ? 0 : div_by(i, nb, rcp);
        const int blk = i - row[p] * nb;
        col[p] = blk * ROW8_BLOCK + lane * V;
        live[p] = i < n ? a.cols - col[p] : 0;
        if (live[p] > 0) {
          s[p] = a.scales[(row0 + row[p]) * ss + blk];
#pragma unroll
          for (int k = 0; k < N; ++k)
            if (live[p] > k * 16 * V)
              __builtin_memcpy(w[p][k], a.codes + (row0 + row[p]) * cs + col[p] + k * 16 * V, V);
        }
      }
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        if (live[p] <= 0) continue;
        T* y = (T*)a.y + (row0 + row[p]) * a.y_stride + col[p];
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const int left = live[p] - k * 16 * V;
          if (left <= 0) continue;
          float f[V];
#pragma unroll
          for (int e = 0; e < V; e += 4) row8_values4(w[p][k][e / 4], row8_pow2(s[p]), f + e);
          struct {
            T e[V];
          } r;
#pragma unroll
          for (int e = 0; e < V; ++e) r.e[e] = Elem<T>::from_f32(f[e]);
          if (left >= V) {
            store_vector(y + k * 16 * V, r, a.stream);
          } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
              if (e < left) y[k * 16 * V + e] = r.e[e];
          }
        }
      }
    }
  }
}

// A matrix [k][n] in blocks of 128 x 128, a workgroup each: codes as they lie and, through
// LDS, transposed (both products of a matrix read it along their sum).  Bound by latency, load to
// largest magnitude to store: 300 x 300 8.6 us.
template <typename T>
__global__ void __launch_bounds__(256) k_weight8_store(Weight8Args a) {
  constexpr int LS = ROW8_BLOCK + 16;  // a row of the staged block, bytes
  __shared__ __attribute__((aligned(16))) uint8_t tile[ROW8_BLOCK * LS];
  __shared__ uint32_t red[4];
  const int lane = threadIdx.x & 15, group = threadIdx.x >> 4;
  const int kb = blockIdx.y, nb = blockIdx.x;
  const Weight8 w = weight8_parts(a.w8, a.k, a.n);
  Run8<T> x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = kb * ROW8_BLOCK + i * 16 + group, c = nb * ROW8_BLOCK + lane * 8;
    x[i] = load_run<T>((const T*)a.w + (int64_t)min(r, a.k - 1) * a.w_stride + c, r < a.k ? a.n - c : 0);
  }
  // the largest magnitude's bits over the workgroup
  auto over_all = [&](uint32_t m) {
    m = max16(m);
    for (int d = 16; d < 64; d *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
    __syncthreads();
    return max(max(red[0], red[1]), max(red[2], red[3]));
  };
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, largest(x[i]));
  m = over_all(m);
  if (m >= NOT_FINITE) {
    m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      m = max(m, largest_finite(x[i]));
      x[i] = without_infinities(x[i]);
    }
    m = over_all(m);
  }
  const uint32_t s = row8_scale(m);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = i * 16 + group, c = lane * 8;
    const uint2 v = codes_of(x[i], s);
    *(uint2*)(tile + r * LS + c) = v;
    if (kb * ROW8_BLOCK + r < a.k)
      *(uint2*)(w.codes + (int64_t)(kb * ROW8_BLOCK + r) * w.stride + nb * ROW8_BLOCK + c) = v;
  }
  __syncthreads();
  // row n of the transposed matrix: 128 codes by eight threads
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = i * 32 + (threadIdx.x >> 3), k = (threadIdx.x & 7) * 16;
    uint32_t v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v[q] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[q] |= (uint32_t)tile[(k + q * 4 + e) * LS + n] << (8 * e);
    }
    if (nb * ROW8_BLOCK + n < a.n)
      *(uint4*)(w.codes_t + (int64_t)(nb * ROW8_BLOCK + n) * w.stride_t + kb * ROW8_BLOCK + k) =
          uint4{v[0], v[1], v[2], v[3]};
  }
  if (threadIdx.x == 0) {
    w.scales[kb * w.scale_stride + nb] = (uint8_t)s;
    w.scales_t[nb * w.scale_stride_t + kb] = (uint8_t)s;
  }
}

int rows_of_tile(int64_t cols) { return (int)std::max<int64_t>(1, ITEMS / row8_blocks(cols)); }

template <typename K>
hipError_t by_tiles(K kernel, const Rows8Args& a, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  const int R = rows_of_tile(a.cols);
  const int64_t tiles = (a.rows + R - 1) / R;
  hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>(tiles, 1 << 20)), dim3(256), 0, st, a, R, tiles);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rows8_store(bool bf16, const Rows8Args& a, hipStream_t st) {
  return bf16 ? by_tiles(k_rows8_store<__bf16>, a, st) : by_tiles(k_rows8_store<float>, a, st);
}

hipError_t launch_rows8_load(bool bf16, const Rows8Args& a, hipStream_t st) {
  return bf16 ? by_tiles(k_rows8_load<__bf16>, a, st) : by_tiles(k_rows8_load<float>, a, st);
}

hipError_t launch_weight8_store(bool bf16, const Weight8Args& a, hipStream_t st) {
  const dim3 grid((unsigned)row8_blocks(a.n), (unsigned)row8_blocks(a.k));
  if (bf16)
    hipLaunchKernelGGL(k_weight8_store<__bf16>, grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL(k_weight8_store<float>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace sscn
