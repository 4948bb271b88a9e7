// Layer norm of feature rows over their channels, forward and backward.
//
//   mean = sum x / C,  r = 1 / sqrt(sum (x - mean)^2 / C + eps),  h = (x - mean) r
//   forward    y = h gain + shift
//   backward   t = dy gain,  dx = r (t - sum t / C - h sum(t h) / C),
//              dgain = sum over rows of dy h,  dshift = sum over rows of dy
//
// Memory-bound: a row is read once into registers (x, and dy in the backward
// pass), reduced there and written once; the backward pass recomputes mean and r
// from x, which it reads anyway, so no statistics travel between the passes.
// Sums, statistics and parameter gradients are float32.
//
// A row belongs to TPR threads (8 .. 64 of a wave, or a workgroup of 256 .. 1024),
// each holding NV vectors of V elements.  Rows need not be aligned nor their
// length a multiple of V: vectors load from element-aligned addresses, and the
// last one starts V elements before the row's end, where its first `skip`
// elements repeat those of the vector before (they are left out of every sum,
// and stored twice with the same value).

#include "common.h"
#include "kernels.h"
#include "lanes.h"

namespace sscn {

namespace {

template <typename T, int V>
struct Pack {
  T e[V];
};

// V elements from an address aligned to one element
template <typename T, int V>
__device__ inline Pack<T, V> load_pack(const T* p) {
  Pack<T, V> v;
  __builtin_memcpy(&v, p, sizeof(v));
  return v;
}

template <typename T, int V>
__device__ inline void store_pack(T* p, const float (&f)[V]) {
  Pack<T, V> v;
#pragma unroll
  for (int e = 0; e < V; ++e) v.e[e] = Elem<T>::from_f32(f[e]);
  __builtin_memcpy(p, &v, sizeof(v));
}

// Makes the compiler convert a bf16 pack anew behind this point instead of keeping
// its float32 values, which take twice the registers (rows of NV > 1 vectors a
// thread, where registers limit the waves).
template <int NV, typename T, int V>
__device__ inline void keep_packed(Pack<T, V>& p) {
  if constexpr (NV > 1 && sizeof(T) == 2 && V % 2 == 0) {
    uint32_t w[V / 2];
    __builtin_memcpy(w, &p, sizeof(p));
#pragma unroll
    for (int i = 0; i < V / 2; ++i) asm volatile("" : "+v"(w[i]));
    __builtin_memcpy(&p, w, sizeof(p));
  }
}

// Sums of K values over the TPR threads of a row, in all of them.  Rows of more
// than one wave combine their waves in `red` (K x 16 floats), which alternates
// between two buffers: a wave that refills one has passed the barrier that the
// readers of its last contents passed after reading.
template <int TPR, int K>
__device__ inline void row_sums(float (&v)[K], float* red) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = group_sum<(TPR < 64 ? TPR : 64)>(v[k]);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) red[k * 16 + (threadIdx.x >> 6)] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float s = red[k * 16];
#pragma unroll
      for (int w = 1; w < W; ++w) s += red[k * 16 + w];
      v[k] = s;
    }
  }
}

// The columns of a thread's vector i: first column, and how many leading
// elements the vector before it holds already (V or more: the vector is unused).
template <int TPR, int V>
__device__ inline int vec_col(int t, int i, int cols, int& skip) {
  const int at = (t + i * TPR) * V;
  const int c = min(at, cols - V);
  skip = at - c;
  return c;
}

constexpr int threads_of(int tpr) { return tpr < 256 ? 256 : tpr; }

// Forward.  The next row's loads are in flight while a row is reduced; what bounds it
// is memory: 200001 x 100 bf16 in 104-element rows 18.9 us (80 MB, 4.2 TB/s; the caches
// hold part of it), 20011 x 4099 float32 124 .. 129 us (656 MB, 5.1 TB/s: a large copy
// reaches 4.9), a single row 2.7 us of which the launch is 2.4.
template <typename T, int V, int TPR, int NV>
__global__ void __launch_bounds__(threads_of(TPR)) k_norm(NormArgs a) {
  constexpr int NT = threads_of(TPR), RPB = NT / TPR;
  __shared__ float red[2][TPR > 64 ? 16 : 1];
  const int t = threadIdx.x % TPR;
  int col[NV], skip[NV];
  float gain[NV][V], shift[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    col[i] = vec_col<TPR, V>(t, i, a.cols, skip[i]);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      gain[i][e] = a.gain && skip[i] < V ? a.gain[col[i] + e] : 1.f;
      shift[i][e] = a.shift && skip[i] < V ? a.shift[col[i] + e] : 0.f;
    }
  }
  const float rc = 1.f / (float)a.cols;
  const int64_t step = (int64_t)gridDim.x * RPB;
  Pack<T, V> raw[NV], next[NV];
  auto fetch = [&](Pack<T, V>(&to)[NV], int64_t r) {
    const T* x = (const T*)a.x + (a.rmap ? (int64_t)a.rmap[r] : r) * a.x_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (skip[i] < V) to[i] = load_pack<T, V>(x + col[i]);
  };
  int64_t r = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
  if (r < a.rows) fetch(next, r);
  for (; r < a.rows; r += step) {
    // the row stays as loaded and is converted wherever it is used
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      raw[i] = next[i];
#pragma unroll
      for (int e = 0; e < V; ++e) s[0] += e >= skip[i] ? Elem<T>::to_f32(raw[i].e[e]) : 0.f;
    }
    if (r + step < a.rows) fetch(next, r + step);  // in flight while this row is reduced
    row_sums<TPR, 1>(s, red[0]);
    const float mean = s[0] * rc;
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) keep_packed<NV>(raw[i]);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float f = Elem<T>::to_f32(raw[i].e[e]) - mean;
        s[0] += e >= skip[i] ? f * f : 0.f;
      }
    row_sums<TPR, 1>(s, red[1]);
    const float rs = 1.f / sqrtf(s[0] * rc + a.eps);
    T* y = (T*)a.y + r * a.y_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (skip[i] >= V) continue;
      keep_packed<NV>(raw[i]);
      float f[V];
#pragma unroll
      for (int e = 0; e < V; ++e) f[e] = (Elem<T>::to_f32(raw[i].e[e]) - mean) * rs * gain[i][e] + shift[i][e];
      store_pack<T, V>(y + col[i], f);
    }
    for (int c = a.cols + t; c < a.y_cols; c += TPR) y[c] = Elem<T>::from_f32(0.f);
  }
}

// Rows too long for a workgroup's registers: one workgroup a row, read once per
// pass (mean, variance, result) out of the caches.
template <typename T>
__global__ void __launch_bounds__(1024) k_norm_long(NormArgs a) {
  __shared__ float red[2][16];
  const float rc = 1.f / (float)a.cols;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = (const T*)a.x + (a.rmap ? (int64_t)a.rmap[r] : r) * a.x_stride;
    T* y = (T*)a.y + r * a.y_stride;
    float s[1] = {0.f};
    for (int c = threadIdx.x; c < a.cols; c += 1024) s[0] += Elem<T>::to_f32(x[c]);
    row_sums<1024, 1>(s, red[0]);
    const float mean = s[0] * rc;
    s[0] = 0.f;
    for (int c = threadIdx.x; c < a.cols; c += 1024) {
      const float d = Elem<T>::to_f32(x[c]) - mean;
      s[0] += d * d;
    }
    row_sums<1024, 1>(s, red[1]);
    const float rs = 1.f / sqrtf(s[0] * rc + a.eps);
    for (int c = threadIdx.x; c < a.cols; c += 1024)
      y[c] = Elem<T>::from_f32((Elem<T>::to_f32(x[c]) - mean) * rs * (a.gain ? a.gain[c] : 1.f) +
                               (a.shift ? a.shift[c] : 0.f));
    for (int c = a.cols + threadIdx.x; c < a.y_cols; c += 1024) y[c] = Elem<T>::from_f32(0.f);
  }
}

// Backward.  Each thread also sums dy h and dy of its columns over the rows it
// meets; a workgroup writes one partial row of each (part[block][cols], then the
// same for dshift), which k_norm_params adds in a fixed order: no atomics.  Memory-bound:
// 16384 x 8192 bf16 takes 172 us and the parameters' sums 7 (805 MB, 4.7 TB/s; 201 before
// the rows stayed packed in registers), 200001 x 100 bf16 25 and 5 (120 MB, 4.8 TB/s).
template <typename T, typename TD, int V, int TPR, int NV>
__global__ void __launch_bounds__(threads_of(TPR)) k_norm_bwd(NormBwdArgs a) {
  constexpr int NT = threads_of(TPR), RPB = NT / TPR;
  __shared__ float red[2][TPR > 64 ? 48 : 1];
  const int t = threadIdx.x % TPR;
  int col[NV], skip[NV];
  float gain[NV][V], dg[NV][V], ds[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    col[i] = vec_col<TPR, V>(t, i, a.cols, skip[i]);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      gain[i][e] = a.gain && skip[i] < V ? a.gain[col[i] + e] : 1.f;
      dg[i][e] = ds[i][e] = 0.f;
    }
  }
  const float rc = 1.f / (float)a.cols;
  const int64_t step = (int64_t)gridDim.x * RPB;
  Pack<T, V> x[NV], nx[NV];
  Pack<TD, V> d[NV], nd[NV];
  auto fetch = [&](int64_t r) {
    const T* px = (const T*)a.x + (a.rmap ? (int64_t)a.rmap[r] : r) * a.x_stride;
    const TD* pd = (const TD*)a.dy + r * a.dy_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (skip[i] < V) {
        nx[i] = load_pack<T, V>(px + col[i]);
        nd[i] = load_pack<TD, V>(pd + col[i]);
      }
  };
  int64_t r = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
  if (r < a.rows) fetch(r);
  for (; r < a.rows; r += step) {
    // both rows stay as loaded and are converted wherever they are used: fewer
    // registers, so more rows of other workgroups in flight
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      x[i] = nx[i];
      d[i] = nd[i];
#pragma unroll
      for (int e = 0; e < V; ++e) s[0] += e >= skip[i] ? Elem<T>::to_f32(x[i].e[e]) : 0.f;
    }
    if (r + step < a.rows) fetch(r + step);
    row_sums<TPR, 1>(s, red[0]);
    const float mean = s[0] * rc;
    float q[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) keep_packed<NV>(x[i]);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float f = Elem<T>::to_f32(x[i].e[e]) - mean;
        const float tt = Elem<TD>::to_f32(d[i].e[e]) * gain[i][e];
        const bool in = e >= skip[i];
        q[0] += in ? f * f : 0.f;
        q[1] += in ? tt : 0.f;
        q[2] += in ? tt * f : 0.f;
      }
    row_sums<TPR, 3>(q, red[1]);
    const float rs = 1.f / sqrtf(q[0] * rc + a.eps);
    const float m1 = q[1] * rc, m2 = q[2] * rs * rc;
    TD* dx = (TD*)a.dx + r * a.dx_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (skip[i] >= V) continue;
      keep_packed<NV>(x[i]);
      keep_packed<NV>(d[i]);
      float o[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float h = (Elem<T>::to_f32(x[i].e[e]) - mean) * rs, g = Elem<TD>::to_f32(d[i].e[e]);
        o[e] = rs * (g * gain[i][e] - m1 - h * m2);
        dg[i][e] += g * h;
        ds[i][e] += g;
      }
      store_pack<TD, V>(dx + col[i], o);
    }
    for (int c = a.cols + t; c < a.dx_cols; c += TPR) dx[c] = Elem<TD>::from_f32(0.f);
  }
  if (!a.part) return;
  float* pg = a.part + (int64_t)blockIdx.x * a.cols;
  float* ps = pg + (int64_t)gridDim.x * a.cols;
  if constexpr (RPB == 1) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (e >= skip[i] && skip[i] < V) {
          pg[col[i] + e] = dg[i][e];
          ps[col[i] + e] = ds[i][e];
        }
  } else {  // the workgroup's rows in order
    constexpr int WIDTH = TPR * NV * V;
    __shared__ float sum[RPB * WIDTH];
    const int g = threadIdx.x / TPR;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      if (which) __syncthreads();
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (e >= skip[i] && skip[i] < V) sum[g * WIDTH + col[i] + e] = which ? ds[i][e] : dg[i][e];
      __syncthreads();
      for (int c = threadIdx.x; c < a.cols; c += NT) {
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < RPB; ++k) v += sum[k * WIDTH + c];
        (which ? ps : pg)[c] = v;
      }
    }
  }
}

// Rows too long for registers: x and dy are read once per pass, and a thread adds its
// columns' parameter sums to the workgroup's partial row in memory (each column is one
// thread's, so rows are added in order).
template <typename T>
__global__ void __launch_bounds__(1024) k_norm_bwd_long(NormBwdArgs a) {
  using TD = T;
  __shared__ float red[2][48];
  const float rc = 1.f / (float)a.cols;
  float* pg = a.part ? a.part + (int64_t)blockIdx.x * a.cols : nullptr;
  float* ps = a.part ? pg + (int64_t)gridDim.x * a.cols : nullptr;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = (const T*)a.x + (a.rmap ? (int64_t)a.rmap[r] : r) * a.x_stride;
    const TD* dy = (const TD*)a.dy + r * a.dy_stride;
    TD* dx = (TD*)a.dx + r * a.dx_stride;
    float s[1] = {0.f};
    for (int c = threadIdx.x; c < a.cols; c += 1024) s[0] += Elem<T>::to_f32(x[c]);
    row_sums<1024, 1>(s, red[0]);
    const float mean = s[0] * rc;
    float q[3] = {0.f, 0.f, 0.f};
    for (int c = threadIdx.x; c < a.cols; c += 1024) {
      const float f = Elem<T>::to_f32(x[c]) - mean;
      const float tt = Elem<TD>::to_f32(dy[c]) * (a.gain ? a.gain[c] : 1.f);
      q[0] += f * f;
      q[1] += tt;
      q[2] += tt * f;
    }
    row_sums<1024, 3>(q, red[1]);
    const float rs = 1.f / sqrtf(q[0] * rc + a.eps);
    const float m1 = q[1] * rc, m2 = q[2] * rs * rc;
    const bool first = r == blockIdx.x;
    for (int c = threadIdx.x; c < a.cols; c += 1024) {
      const float h = (Elem<T>::to_f32(x[c]) - mean) * rs;
      const float d = Elem<TD>::to_f32(dy[c]);
      if (pg) {  // this thread's own columns
        pg[c] = (first ? 0.f : pg[c]) + d * h;
        ps[c] = (first ? 0.f : ps[c]) + d;
      }
      dx[c] = Elem<TD>::from_f32(rs * (d * (a.gain ? a.gain[c] : 1.f) - m1 - h * m2));
    }
    for (int c = a.cols + threadIdx.x; c < a.dx_cols; c += 1024) dx[c] = Elem<TD>::from_f32(0.f);
  }
}

// dgain (blockIdx.y = 0) and dshift (1): the partials of 64 columns, in 16
// interleaved slices combined in order, 16 loads of a slice in flight: 1024 partial
// rows of 100 columns take 5.4 us (latency), 512 of 8192 columns 7.0.
__global__ void __launch_bounds__(1024) k_norm_params(const float* __restrict__ part, int parts, int cols, float* dgain,
                                                      float* dshift) {
  __shared__ float red[16][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), sl = threadIdx.x >> 6;
  float* out = blockIdx.y ? dshift : dgain;
  const float* p = part + (blockIdx.y ? (int64_t)parts * cols : 0);
  float v = 0.f;
  if (c < cols)
#pragma unroll 16
    for (int k = sl; k < parts; k += 16) v += p[(int64_t)k * cols + c];
  red[sl][threadIdx.x & 63] = v;
  __syncthreads();
  if (sl == 0 && c < cols && out) {
    for (int k = 1; k < 16; ++k) v += red[k][threadIdx.x];
    out[c] = v;
  }
}

// The shape that a row length takes.
struct NormShape {
  int tpr, nv;  // tpr 0: the looping kernel
  bool scalar;  // fewer columns than a vector holds
  int rpb() const { return tpr == 0 ? 1 : threads_of(tpr) / tpr; }
};

// two: rows of up to 64 vectors in half the lanes, two vectors a lane.
NormShape norm_shape(int ve, int cols, bool two) {
  if (cols < ve) return {8, 1, true};
  const int nvec = (cols + ve - 1) / ve;
  if (two && nvec > 8 && nvec <= 64) return {nvec <= 16 ? 8 : nvec <= 32 ? 16 : 32, 2, false};
  if (nvec <= 8) return {8, 1, false};
  if (nvec <= 16) return {16, 1, false};
  if (nvec <= 32) return {32, 1, false};
  if (nvec <= 64) return {64, 1, false};
  if (nvec <= 128) return {64, 2, false};
  if (nvec <= 256) return {256, 1, false};
  if (nvec <= 512) return {256, 2, false};
  if (nvec <= 1024) return {512, 2, false};
  if (nvec <= 2048) return {1024, 2, false};
  return {0, 0, false};
}

// float32 gradients of bf16 rows come from the softmax layer only, whose input has at
// most 256 vectors a row (sscn_net_create refuses wider layers)
constexpr int HEAD_VECS = 256;

int64_t row_blocks(const NormShape& s, int64_t rows) { return (rows + s.rpb() - 1) / s.rpb(); }

template <typename T>
hipError_t norm_fwd(const NormArgs& a, hipStream_t st) {
  constexpr int VE = Elem<T>::VE;
  // where rows abound, more bytes in flight (200001 rows of 100 bf16: 18.8 us with two
  // vectors a lane, 21.1 with one; a single row of 300: 7.7 with one, 8.3 with two)
  const NormShape s = norm_shape(VE, a.cols, a.rows >= 8192);
  const int grid = (int)std::min<int64_t>(row_blocks(s, a.rows), s.tpr == 0 || s.tpr == 1024 ? 512 : s.tpr == 512 ? 1024 : 2048);
#define SSCN_NORM(V, TPR, NV) \
  case TPR * 8 + NV: hipLaunchKernelGGL((k_norm<T, V, TPR, NV>), dim3(grid), dim3(threads_of(TPR)), 0, st, a); break
  if (s.tpr == 0)
    hipLaunchKernelGGL(k_norm_long<T>, dim3(grid), dim3(1024), 0, st, a);
  else if (s.scalar)
    hipLaunchKernelGGL((k_norm<T, 1, 8, 1>), dim3(grid), dim3(256), 0, st, a);
  else
    switch (s.tpr * 8 + s.nv) {
      SSCN_NORM(VE, 8, 1);
      SSCN_NORM(VE, 8, 2);
      SSCN_NORM(VE, 16, 1);
      SSCN_NORM(VE, 16, 2);
      SSCN_NORM(VE, 32, 1);
      SSCN_NORM(VE, 32, 2);
      SSCN_NORM(VE, 64, 1);
      SSCN_NORM(VE, 64, 2);
      SSCN_NORM(VE, 256, 1);
      SSCN_NORM(VE, 256, 2);
      SSCN_NORM(VE, 512, 2);
      SSCN_NORM(VE, 1024, 2);
      default: return hipErrorInvalidValue;
    }
#undef SSCN_NORM
  return hipGetLastError();
}

template <typename T, typename TD>
hipError_t norm_bwd(const NormBwdArgs& a, int grid, hipStream_t st) {
  constexpr int VE = Elem<T>::VE;
  const NormShape s = norm_shape(VE, a.cols, false);
#define SSCN_NORM(V, TPR, NV)                                                                                     \
  case TPR * 8 + NV:                                                                                              \
    if constexpr (sizeof(T) == sizeof(TD) || TPR * NV <= HEAD_VECS)                                               \
      hipLaunchKernelGGL((k_norm_bwd<T, TD, V, TPR, NV>), dim3(grid), dim3(threads_of(TPR)), 0, st, a);           \
    else                                                                                                          \
      return hipErrorInvalidValue;                                                                                \
    break
  if (sizeof(T) != sizeof(TD) && (s.tpr == 0 || s.tpr * s.nv > HEAD_VECS)) return hipErrorInvalidValue;
  if constexpr (sizeof(T) == sizeof(TD))
    if (s.tpr == 0) {
      hipLaunchKernelGGL(k_norm_bwd_long<T>, dim3(grid), dim3(1024), 0, st, a);
      return hipGetLastError();
    }
  if (s.scalar)
    hipLaunchKernelGGL((k_norm_bwd<T, TD, 1, 8, 1>), dim3(grid), dim3(256), 0, st, a);
  else
    switch (s.tpr * 8 + s.nv) {
      SSCN_NORM(VE, 8, 1);
      SSCN_NORM(VE, 16, 1);
      SSCN_NORM(VE, 32, 1);
      SSCN_NORM(VE, 64, 1);
      SSCN_NORM(VE, 64, 2);
      SSCN_NORM(VE, 256, 1);
      SSCN_NORM(VE, 256, 2);
      SSCN_NORM(VE, 512, 2);
      SSCN_NORM(VE, 1024, 2);
      default: return hipErrorInvalidValue;
    }
#undef SSCN_NORM
  return hipGetLastError();
}

}  // namespace

int64_t norm_parts(bool bf16, int64_t rows, int32_t cols) {
  // (one vector a lane: its sums double the registers; 200001 rows of 100 bf16: 30.5 us, 33.3 with two)
  const NormShape s = norm_shape(bf16 ? 8 : 4, cols, false);
  // as many workgroups as the compute units hold at once: 16 waves each
  const int64_t fill = s.tpr == 0 || s.tpr == 1024 ? 256 : s.tpr == 512 ? 512 : 1024;
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(fill, ((int64_t)1 << 25) / cols));
  return std::max<int64_t>(1, std::min(row_blocks(s, rows), most));
}

hipError_t launch_norm(bool bf16, const NormArgs& a, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  return bf16 ? norm_fwd<__bf16>(a, st) : norm_fwd<float>(a, st);
}

hipError_t launch_norm_bwd(bool bf16, bool f32_grads, const NormBwdArgs& a, float* dgain, float* dshift, hipStream_t st) {
  if (a.rows <= 0) {  // sums over nothing
    hipError_t e = dgain ? launch_fill_zero(dgain, (int64_t)a.cols * 4, st) : hipSuccess;
    return e == hipSuccess && dshift ? launch_fill_zero(dshift, (int64_t)a.cols * 4, st) : e;
  }
  const int grid = (int)norm_parts(bf16, a.rows, a.cols);
  const hipError_t e = !bf16       ? norm_bwd<float, float>(a, grid, st)
                       : f32_grads ? norm_bwd<__bf16, float>(a, grid, st)
                                   : norm_bwd<__bf16, __bf16>(a, grid, st);
  if (e != hipSuccess || !a.part) return e;
  hipLaunchKernelGGL(k_norm_params, dim3((a.cols + 63) / 64, 2), dim3(1024), 0, st, (const float*)a.part, grid, a.cols,
                     dgain, dshift);
  return hipGetLastError();
}

}  // namespace sscn
