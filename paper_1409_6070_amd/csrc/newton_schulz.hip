// Orthogonalising matrices by Newton-Schulz products, and the weight update that
// uses the result (Muon).
//
//   X = u / |u|_F  (m x n with m <= n: transposed where u is taller than wide)
//   each step:  A = X X^T,  B = b A + c A A,  X <- a X + B X
//
// The odd polynomial p(s) = a s + b s^3 + c s^5 acts on X's singular values and
// leaves its singular vectors: a few steps bring all but the smallest near 1.
//
// Precision.  X is kept in float32.  A product's operands, A and B among them, are
// split into two fp16 numbers each, hi + lo, and multiplied on the fp16 matrix cores
// as hi hi + hi lo + lo hi with float32 sums: three times the matrix work of a plain
// fp16 product, which the fp16 cores still do at five times the rate of float32 MFMA
// (4096 x 4096: 383 TFLOP/s of the formula's operations; a library's float32 product
// reaches 154).  An operand is scaled by the power of two that brings the largest value
// it may hold near fp16's end (NsStep).  An entry is then off by 2^-22 of itself or,
// where its lo part falls below fp16's smallest step, by 2^-39 of that largest value.
// A small singular value is carried from step to step by a X alone (B's rows along it
// are small), which is float32 throughout: relative to the matrix the result is as
// near to the formula's as a float32 computation's, where operands of fewer bits lose
// the small singular values, whose errors every step multiplies by a (about 3.4).  A
// row or column far smaller than the others is less exact relative to itself, since the
// scales are the matrix's: every second row (column) of 300 x 1000 at 1e-4 of the others
// is off by 1.7e-7 (1.3e-6), at 1e-6 by 1.4e-6 (3.5e-5); float32 products 2.9e-7 (2.3e-6)
// at either.
//
// Layout.  An operand with R rows of K values is stored as the matrix cores read
// it: blocks of 16 rows x 32 k, row-block major, a block's hi plane of 1 KiB then
// its lo plane, lane l's 16 bytes being row l % 16, k 8 (l / 16) .. + 7.  One wave
// moves a plane with one 16-byte load per lane straight into LDS and reads it
// back the same way: contiguous everywhere, no bank conflicts, no swizzle.  Rows
// and columns are padded with zeros to multiples of 32.

#include <atomic>
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace sscn {

static_assert(sizeof(NsGroup) + 128 <= 4096, "kernel arguments must fit the 4 KiB argument segment");

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int BLOCK = 2048;  // bytes of a 16 x 32 block, both planes

// s_waitcnt vmcnt(n) lgkmcnt(0)
template <int N>
__device__ inline void wait_loads() {
  static_assert(N >= 0 && N < 64, "vmcnt field");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
}

// One 16-byte load per lane into LDS: lane l's bytes, lane_off + off into the buffer,
// land at lds + 16 l (lds and off uniform over the wave).  The compiler does not see
// it; wait_loads and the barriers' fences order it.
__device__ inline void load_plane(u32x4 rsrc, uint32_t lds, uint32_t lane_off, uint32_t off) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds),
      "v"(lane_off), "s"(rsrc), "s"(off)
      : "m0");
}

__device__ inline u32x4 plane_rsrc(const void* base, uint32_t bytes) {
  const uint64_t b = (uint64_t)base;
  return u32x4{(uint32_t)b, (uint32_t)(b >> 32) & 0xffffu, bytes, 0x00020000u};
}

__device__ inline uint32_t lds_offset(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// Eight values as hi and lo planes: 16 bytes each, 1 KiB apart.
__device__ inline void store_split(char* at, const float (&v)[8], float s) {
  f16x8 hi, lo;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float x = v[e] * s;
    hi[e] = (_Float16)x;
    lo[e] = (_Float16)(x - (float)hi[e]);
  }
  *(f16x8*)at = hi;
  *(f16x8*)(at + BLOCK / 2) = lo;
}

// Address of lane l's part of block (rb, kb) of an operand with kblocks blocks a row.
__device__ inline int64_t block_at(int rb, int kb, int kblocks) { return ((int64_t)rb * kblocks + kb) * BLOCK; }

// Matrix j, its pointers known to be global memory's.  Out of a table in memory the
// compiler takes them for flat ones, whose loads share a counter with LDS and return in
// any order: it then waits for all of them wherever one is needed.
template <typename T>
__device__ inline T* global_pointer(T* const& p) {
  return (T*)*(__attribute__((address_space(1))) T* const*)&p;
}
__device__ inline NsMat matrix(const NsTable* t, int j) {
  const NsMat& from = t->mat[j];
  NsMat M = from;
  M.X = global_pointer(from.X);
  M.opX = global_pointer(from.opX);
  M.opXt[0] = global_pointer(from.opXt[0]);
  M.opXt[1] = global_pointer(from.opXt[1]);
  M.opA = global_pointer(from.opA);
  M.opB = global_pointer(from.opB);
  M.ssq = global_pointer(from.ssq);
  M.u = global_pointer(from.u);
  M.o = global_pointer(from.o);
  M.w = global_pointer(from.w);
  M.v = global_pointer(from.v);
  return M;
}

__device__ inline int find_mat(const NsArgs& a, int t) {
  int j = 0;
  while (j + 1 < a.n && t >= a.beg[j + 1]) ++j;
  return j;
}

// The kernels of a product, by its 128 x 128 tiles, their slabs of 32 k per compute unit
// and its 64 x 64 tiles, as plan_product counts them.  Measured, us, 128 / 64 / 32 tiles:
//   X X^T  2100 x 3900 (73 slabs)  76 / 86 / -;  2048 x 2048 (34)  44 / 46 / -;  1800 x 1900 (28)
//          41.7 / 31.5 / -;  1500 x 1500 (14; 300 tiles of 64)  31.7 / 21.0 / 33.4;  1300 x 1300
//          (231)  27.1 / 14.0 / 23.4;  1100 x 1100 (171)  - / 12.0 / 14.2;  1000 x 600 three times
//          (165)  24.8 / 14.0 / 12.5;  1000 x 300 (15)  17.0 / 10.0 / 6.3
//          lists with a softmax matrix (3755 columns, four times the others' sums):
//          DeepCNet(6,100) (24; 277)  39.7 / 36.0 / 35.2;  DeepCNet(5,100) (200)  - / 26.4 / 27.5;
//          DeepCNiN(6,55) (196)  - / 24.6 / 18.6;  DeepCNiN(5,65) (194)  - / 24.4 / 18.1;
//          DeepCNet(5,90) (169)  - / 25.1 / 23.0;  DeepCNiN(5,50) (105)  27.3 / 23.2 / 14.8
//   B X    1500 x 1500 (26 slabs)  36.5 / 42.5 / 63.9;  1300 x 1300 (19)  38.2 / 25.4 / 43.5;
//          400 x 1600 four times (208 tiles of 128)  21.2 / 28.0 / 23.4;  700 x 3755 (180)  24.4 / 32.4 /
//          38.9;  1000 x 600 three times (120; 480 of 64)  32.8 / 18.8 / 20.4;  2047 x 822 (112; 416)  34.4 /
//          20.9 / 30.0;  1000 x 1000 (64; 256)  - / 14.0 / 19.4;  DeepCNet(5,50) (59; 202)  17.8 / 11.4 / 9.4
// NS_TILES_64 lies where matrices of like sums cross.  The rule does not see that some
// sums are longer: lists like DeepCNiN(5,65)'s, whose 64 x 64 tiles wait for their longest
// sums, are up to 6 us a product slower than in 32 x 32 tiles.
constexpr int NS_CUS = 256, NS_SLABS = 30, NS_SLABS_APPLY = 20, NS_TILES_APPLY = 160, NS_TILES_64 = 170,
              NS_TILES_64_APPLY = 256, NS_FULL = 192;
constexpr int NS_PARTS = 16;  // workgroups that share a tile, at most

// Sum over the workgroup's 256 threads, in all of them (red: four doubles).
__device__ inline double block_sum(double s, double* red) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// ---------------------------------------------------------------------------
// |u|_F^2 as partial sums in float64 (any float32 matrix's fits), and for Muon
// the velocity: v <- mu v + g.  NS_SSQ workgroups at most per matrix; the loads of
// eight elements a thread are in flight together.  Memory-bound where the matrix is
// large (4096 x 4096: 15.3 us, 4.4 TB/s), else one load's latency and the launch
// (1000 x 300: 3.7 us).
//
// The first launch of a group: it also copies the table and clears the counters.
template <typename T, bool MUON>
__global__ void __launch_bounds__(256) k_ns_begin(NsArgs a, NsTable t) {
  constexpr int U = 8;
  if (blockIdx.x == 0) {
    for (int i = threadIdx.x; i < NS_COUNT; i += 256) a.count[i] = 0;
    // from the argument segment, where t lies behind a
    constexpr int AT = (sizeof(NsArgs) + alignof(NsTable) - 1) / alignof(NsTable) * alignof(NsTable);
    const auto* from = (const __attribute__((address_space(4))) uint32_t*)(
        (const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr() + AT);
    for (int i = threadIdx.x; i < (int)(sizeof(NsTable) / 4); i += 256) ((uint32_t*)a.table)[i] = from[i];
  }
  const int j = find_mat(a, blockIdx.x);
  const NsMat M = matrix(&t, j);
  const int blk = blockIdx.x - a.beg[j], nblk = a.beg[j + 1] - a.beg[j];
  const int64_t rows = M.tall ? M.n : M.m, cols = M.tall ? M.m : M.n, total = rows * cols;
  double s = 0.0;
  if (MUON || M.u_stride == cols) {
    const T* u = (const T*)M.u;
    const int64_t step = (int64_t)nblk * 256;
    for (int64_t i0 = (int64_t)blk * 256 + threadIdx.x; i0 < total; i0 += U * step) {
      float x[U], v[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {  // (past the end: the last element, not used)
        const int64_t i = std::min(i0 + k * step, total - 1);
        x[k] = Elem<T>::to_f32(u[i]);
        if constexpr (MUON) v[k] = M.v[i];
      }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int64_t i = i0 + k * step;
        if constexpr (MUON) {
          v[k] = a.momentum * v[k] + x[k];
          if (i < total) M.v[i] = v[k];
          x[k] = a.nesterov ? a.momentum * v[k] + x[k] : v[k];
        }
        s += i < total ? (double)x[k] * x[k] : 0.0;
      }
    }
  } else {
    const T* u = (const T*)M.u;
    int tx = 256;  // threads along a row: short rows go several at a time
    while (tx / 2 >= cols) tx /= 2;
    const int64_t step = (int64_t)nblk * (256 / tx);
    for (int64_t c = threadIdx.x % tx; c < cols; c += tx)
      for (int64_t r0 = (int64_t)blk * (256 / tx) + threadIdx.x / tx; r0 < rows; r0 += U * step) {
        float x[U];
#pragma unroll
        for (int k = 0; k < U; ++k) x[k] = Elem<T>::to_f32(u[std::min(r0 + k * step, rows - 1) * M.u_stride + c]);
#pragma unroll
        for (int k = 0; k < U; ++k) s += r0 + k * step < rows ? (double)x[k] * x[k] : 0.0;
      }
  }
  __shared__ double red[4];
  s = block_sum(s, red);
  if (threadIdx.x == 0) M.ssq[blk] = s;
}

// X = u / |u|_F in float32 and as both operands; a wave per 32 x 32 tile, whose
// values are on their way while the norm's partial sums are added (7 us instead of
// 13 at 1000 x 300).  Reads 4 bytes an element and writes 12: 4096 x 4096 takes
// 46 us, 5.8 TB/s.
template <typename T, bool MUON>
__global__ void __launch_bounds__(256) k_ns_convert(NsArgs a) {
  const int j = find_mat(a, blockIdx.x);
  const NsMat M = matrix(a.table, j);
  __shared__ double red[4];
  __shared__ float tile[4][32][36];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int tn = M.np / 32, t = (blockIdx.x - a.beg[j]) * 4 + wave;
  const bool live = t < (M.mp / 32) * tn;
  const int i0 = live ? t / tn * 32 : 0, j0 = live ? t % tn * 32 : 0;
  // lanes along the caller's rows; outside the matrix a lane reads its nearest element
  const int64_t stride = MUON ? (M.tall ? M.m : M.n) : M.u_stride;
  const int r0 = M.tall ? j0 : i0, c = (M.tall ? i0 : j0) + (lane & 31), p0 = lane >> 5;
  const int rows = M.tall ? M.n : M.m, cols = M.tall ? M.m : M.n;
  const int64_t at0 = std::min(c, cols - 1);
  float x[16], v[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const int64_t at = std::min(r0 + p0 + 2 * k, rows - 1) * stride + at0;
    if constexpr (MUON) {
      v[k] = M.v[at];
      x[k] = ((const float*)M.u)[at];
    } else {
      x[k] = Elem<T>::to_f32(((const T*)M.u)[at]);
    }
  }
  double ss = 0.0;
  for (int k = threadIdx.x; k < M.nssq; k += 256) ss += M.ssq[k];
  ss = block_sum(ss, red);
  const double inv = ss == 0.0 ? 0.0 : 1.0 / sqrt(ss);  // (a zero matrix stays zero)
  // the padding stays zero, beside a matrix whose norm is NaN or infinite too
  float* to = M.tall ? &tile[wave][lane & 31][p0] : &tile[wave][p0][lane & 31];
  const int ts = M.tall ? 2 : 2 * 36;
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    if constexpr (MUON) x[k] = a.nesterov ? a.momentum * v[k] + x[k] : v[k];
    to[k * ts] = c < cols && r0 + p0 + 2 * k < rows ? (float)((double)x[k] * inv) : 0.f;
  }
  __syncthreads();
  if (!live) return;
  const int r16 = lane & 15, k8 = lane >> 4;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float w[8];
    const int i = h * 16 + r16;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = tile[wave][i][k8 * 8 + e];
    float* X = M.X + (int64_t)(i0 + i) * M.np + j0 + k8 * 8;
    *(f32x4*)X = f32x4{w[0], w[1], w[2], w[3]};
    *(f32x4*)(X + 4) = f32x4{w[4], w[5], w[6], w[7]};
    store_split(M.opX + block_at(i0 / 16 + h, j0 / 32, M.np / 32) + lane * 16, w, a.scale);
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = tile[wave][k8 * 8 + e][h * 16 + r16];
    store_split(M.opXt[0] + block_at(j0 / 16 + h, i0 / 32, M.mp / 32) + lane * 16, w, a.scale);
  }
}

// ---------------------------------------------------------------------------
// the products: C[i][j] = sum_k P[i][k] Q[j][k]

enum NsKind { NS_GRAM, NS_POLY, NS_APPLY, NS_ORTHO, NS_MUON };

constexpr bool symmetric(int kind) { return kind == NS_GRAM || kind == NS_POLY; }

// A TM x TN result tile: its matrix, place and operands.
template <int TM, int TN, int KIND>
struct NsWork {
  static_assert(TM % TN == 0, "a tile row is one or several tile columns high");
  NsMat M;
  int ti, tj;       // tile row and column
  int kblocks;        // blocks of k in the operands' rows
  int k0, k1;         // those of this workgroup
  int part, parts;    // which of the workgroups that share the tile
  int slot, counter;  // the tile's first partial tile, its counter
  const char *P, *Q;  // first block of the tile's rows in each operand
  char *Xt, *Xt_next; // this step's operand with X's columns, and the next one's
  int pr, qr;         // row blocks of each inside the padded matrix (a last tile has fewer)

  // false: no tile for this workgroup.  Workgroup b runs on XCD b % 8: each XCD takes
  // an eighth of every matrix's tiles, rounded up, consecutive ones, whose operands its
  // L2 shares; the last XCDs take what is left (X X^T of eight 1024 x 1024: 40 tiles on
  // seven of them, 8 on the last).
  __device__ inline bool find(const NsArgs& a) {
    const int xcd = blockIdx.x & 7, slot_of_xcd = blockIdx.x >> 3;
    const int j = find_mat(a, slot_of_xcd);
    M = matrix(a.table, j);
    const NsDeal D = a.deal[j];
    Xt = a.step % 2 ? M.opXt[1] : M.opXt[0];
    Xt_next = a.step % 2 ? M.opXt[0] : M.opXt[1];
    const int tm = (M.mp + TM - 1) / TM, whole = (D.whole + 7) / 8;
    int t = slot_of_xcd - a.beg[j];
    part = 0;
    parts = 1;
    if (t < whole) {
      t += xcd * whole;
      if (t >= D.whole) return false;
    } else {
      const int r = xcd * (a.beg[j + 1] - a.beg[j] - whole) + t - whole, q = r / D.parts;
      t = D.whole + q;
      part = r - q * D.parts;
      parts = D.parts;
      slot = D.slot + q * D.parts;
      counter = D.counter + q;
    }
    if constexpr (symmetric(KIND)) {  // tiles that reach the diagonal or lie below it
      constexpr int R = TM / TN;
      ti = 0;  // R (1 + 2 + .. + ti) tiles in the rows above
      ti = (int)((sqrtf(8.f / R * (float)t + 1.f) - 1.f) * 0.5f);
      while (R * ti * (ti + 1) / 2 > t) --ti;
      while (R * (ti + 1) * (ti + 2) / 2 <= t) ++ti;
      tj = t - R * ti * (ti + 1) / 2;
    } else {
      const int tn = (M.np + TN - 1) / TN;
      ti = t / tn;
      tj = t - ti * tn;
    }
    ti = __builtin_amdgcn_readfirstlane(ti);
    tj = __builtin_amdgcn_readfirstlane(tj);
    const int mp = M.mp, cols = symmetric(KIND) ? mp : M.np;
    if (ti >= tm || tj * TN >= cols) return false;
    kblocks = (KIND == NS_GRAM ? M.np : mp) / 32;
    k0 = kblocks * part / parts;
    k1 = kblocks * (part + 1) / parts;
    P = KIND == NS_GRAM ? M.opX : KIND == NS_POLY ? M.opA : M.opB;
    Q = KIND == NS_GRAM ? M.opX : KIND == NS_POLY ? M.opA : Xt;
    P += block_at(ti * (TM / 16), 0, kblocks);
    Q += block_at(tj * (TN / 16), 0, kblocks);
    pr = min(TM, mp - ti * TM) / 16;
    qr = min(TN, cols - tj * TN) / 16;
    return true;
  }

  // Of a symmetric result, the part of row block rb: 1 below the diagonal's squares
  // of edge TN (stored, and mirrored), 0 on it (stored), -1 above (another's mirror).
  __device__ inline int side(int rb) const {
    if constexpr (!symmetric(KIND)) return 1;
    const int d = ti * (TM / TN) + rb * 16 / TN - tj;
    return d > 0 ? 1 : d == 0 ? 0 : -1;
  }
};

// What the epilogue reads at a 16 x 32 block beside the sums, lane l's part (row
// l % 16, columns 8 (l / 16) .. + 7): A's planes (POLY), X's values (APPLY and the
// last ones), 16 bytes at each of two addresses.
template <class W, int KIND>
__device__ inline const char* beside_at(const W& w, int row16, int col32, int lane, int half) {
  if constexpr (KIND == NS_POLY)
    return w.M.opA + block_at(row16, col32, w.M.mp / 32) + lane * 16 + half * (BLOCK / 2);
  else
    return (const char*)(w.M.X + (int64_t)(row16 * 16 + (lane & 15)) * w.M.np + col32 * 32 + (lane >> 4) * 8 + half * 4);
}

// ... straight into LDS (2 KiB at lds), waited for with wait_loads.
template <class W, int KIND>
__device__ inline void load_beside(const W& w, int row16, int col32, int lane, uint32_t lds) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %1, off" ::"s"(lds + h * 1024),
        "v"(beside_at<W, KIND>(w, row16, col32, lane, h))
        : "m0");
}

template <int KIND>
__device__ inline void beside_values(u32x4 p, u32x4 q, float (&x)[8]) {
  if constexpr (KIND == NS_POLY) {
    const f16x8 hi = __builtin_bit_cast(f16x8, p), lo = __builtin_bit_cast(f16x8, q);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)hi[e] + (float)lo[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = __uint_as_float(p[e]);
      x[4 + e] = __uint_as_float(q[e]);
    }
  }
}

// Eight consecutive elements of a row of the caller's array, from column c on, of
// which the first n exist (n <= 0: none); addresses aligned to one element.
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
    for (int e = 0; e < 8; ++e) r.e[e] = e < n ? p[e] : T(0);
  }
  return r;
}
template <typename T>
__device__ inline void store_run(T* p, const float (&v)[8], int n) {
  Run8<T> r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r.e[e] = Elem<T>::from_f32(v[e]);
  if (n >= 8) {
    __builtin_memcpy(p, &r, sizeof(r));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = r.e[e];
  }
}

// Row `row` of the caller's matrix, columns c .. c + 7: the orthogonal matrix, or the
// weights it updates (their old values in `old`).
template <int KIND, typename TO>
__device__ inline void store_result(const NsMat& M, int row, int c, const float (&o)[8], const Run8<float>& old) {
  const int rows = M.tall ? M.n : M.m, cols = M.tall ? M.m : M.n;
  const int n = row < rows ? cols - c : 0;
  if constexpr (KIND == NS_ORTHO) {
    store_run<TO>((TO*)M.o + (int64_t)row * M.o_stride + c, o, n);
  } else {
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = old.e[e] - (M.scale * o[e] + M.decay * old.e[e]);
    const int64_t at = (int64_t)row * cols + c;
    store_run<float>(M.w + at, w, n);
    if (M.o) store_run<TO>((TO*)M.o + at, w, n);
  }
}
template <int KIND>
__device__ inline Run8<float> load_weights(const NsMat& M, int row, int c) {
  if constexpr (KIND != NS_MUON) return Run8<float>{};
  const int rows = M.tall ? M.n : M.m, cols = M.tall ? M.m : M.n;
  return load_run<float>(M.w + (int64_t)row * cols + c, row < rows ? cols - c : 0);
}

// A tile that several workgroups share: each stores its sums (staged in LDS) as a
// partial tile; the last one to finish adds them all in their order, back into LDS,
// and returns true.  Every wave's stores are in L2 before the barrier; thread 0 then
// releases them with the counter, and the last acquires.
template <int TM, int TN, int NT, class W>
__device__ inline bool join_parts(const NsArgs& a, const W& w, float* Cs) {
  constexpr int CS = TN + 4, V = TM * TN / 4;
  static_assert(V % NT == 0, "whole vectors per thread");
  __shared__ int last;
  f32x4* out = (f32x4*)(a.part + (int64_t)(w.slot + w.part) * (TM * TN));
  for (int i = threadIdx.x; i < V; i += NT)
    out[i] = *(const f32x4*)(Cs + i / (TN / 4) * CS + i % (TN / 4) * 4);
  // Waits in asm, for the stores (the barrier alone waits for none) and for the write-back:
  // behind a wait that it knows of the compiler takes nothing to be outstanding, and
  // leaves out its own between the write-back and the counter.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    last = __hip_atomic_fetch_add(a.count + w.counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == w.parts - 1;
  }
  __syncthreads();
  if (!last) return false;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  const f32x4* in = (const f32x4*)(a.part + (int64_t)w.slot * (TM * TN)) + threadIdx.x;
  constexpr int N = V / NT;  // a part's loads are in flight together
  f32x4 sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) sum[i] = in[i * NT];
#pragma unroll 1
  for (int p = 1; p < w.parts; ++p) {
    f32x4 more[N];
#pragma unroll
    for (int i = 0; i < N; ++i) more[i] = in[(int64_t)p * V + i * NT];
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] += more[i];
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int at = threadIdx.x + i * NT;
    *(f32x4*)(Cs + at / (TN / 4) * CS + at % (TN / 4) * 4) = sum[i];
  }
  if (threadIdx.x == 0) __hip_atomic_store(a.count + w.counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  return true;
}

// The tile's sums, staged in LDS as PARTS partial tiles [TM][TN + 4], to the result:
// first along the rows, then along the columns, in blocks of 16 x 32 dealt to NW
// waves, GROUP blocks at a time whose reads are in flight together.  With PRE,
// `beside` holds what load_beside brought for each block.
template <int TM, int TN, int KIND, typename TO, int NW, int PARTS, int GROUP, bool PRE>
__device__ inline void finish_tile(const NsArgs& a, const NsWork<TM, TN, KIND>& w, float* Cs, int wave, int lane,
                                   const char* beside) {
  using W = NsWork<TM, TN, KIND>;
  constexpr int CS = TN + 4;
  constexpr bool LAST = KIND == NS_ORTHO || KIND == NS_MUON;
  const NsMat& M = w.M;
  const int l16 = lane & 15, g4 = lane >> 4;
  {
    constexpr int KB = TN / 32, NB = TM / 16 * KB, PER = (NB + NW - 1) / NW, G = GROUP < PER ? GROUP : PER;
    const int row0 = w.ti * (TM / 16), col0 = w.tj * KB;
#pragma unroll 1
    for (int n0 = 0; n0 < PER; n0 += G) {
      u32x4 bes[G][2];
      Run8<float> old[G];
#pragma unroll
      for (int g = 0; g < G; ++g) {  // (blocks outside the matrix: the nearest one, not used)
        const int b = min(wave + (n0 + g) * NW, NB - 1), rb = min(b / KB, w.pr - 1), kb = min(b % KB, w.qr / 2 - 1);
        if constexpr (KIND != NS_GRAM) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
            bes[g][h] = *(const u32x4*)(PRE ? beside + (rb * KB + kb) * 2048 + h * 1024 + lane * 16
                                            : beside_at<W, KIND>(w, row0 + rb, col0 + kb, lane, h));
        }
        if (KIND == NS_MUON && !M.tall)
          old[g] = load_weights<KIND>(M, (row0 + rb) * 16 + l16, (col0 + kb) * 32 + g4 * 8);
      }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const int b = wave + (n0 + g) * NW, rb = b / KB, kb = b % KB;
        if (n0 + g >= PER || b >= NB || rb >= w.pr || 2 * kb >= w.qr || w.side(rb) < 0) continue;
        float* c = Cs + (rb * 16 + l16) * CS + kb * 32 + g4 * 8;
        float v[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          f32x4 s = *(const f32x4*)(c + 4 * h);
#pragma unroll
          for (int p = 1; p < PARTS; ++p) s += *(const f32x4*)(c + 4 * h + p * TM * CS);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[4 * h + e] = s[e] * a.of_sum;
        }
        float x[8];
        if constexpr (KIND != NS_GRAM) {
          beside_values<KIND>(bes[g][0], bes[g][1], x);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = fmaf(a.of_beside, x[e], v[e]);
        }
        if constexpr (KIND == NS_GRAM) {
          store_split(M.opA + block_at(row0 + rb, col0 + kb, M.mp / 32) + lane * 16, v, a.scale);
        } else if constexpr (KIND == NS_POLY) {
          store_split(M.opB + block_at(row0 + rb, col0 + kb, M.mp / 32) + lane * 16, v, a.scale);
        } else {
          if constexpr (KIND == NS_APPLY) {
            float* X = M.X + (int64_t)((row0 + rb) * 16 + l16) * M.np + (col0 + kb) * 32 + g4 * 8;
            *(f32x4*)X = *(const f32x4*)v;
            *(f32x4*)(X + 4) = *(const f32x4*)(v + 4);
            store_split(M.opX + block_at(row0 + rb, col0 + kb, M.np / 32) + lane * 16, v, a.scale);
          } else if (!M.tall) {
            store_result<KIND, TO>(M, (row0 + rb) * 16 + l16, (col0 + kb) * 32 + g4 * 8, v, old[g]);
          }
        }
        *(f32x4*)c = *(const f32x4*)v;
        *(f32x4*)(c + 4) = *(const f32x4*)(v + 4);
      }
    }
  }
  if (LAST && !M.tall) return;
  __syncthreads();
  // the mirrored part of a symmetric result, X's other operand, or a tall result
  constexpr int KB = TM / 32, NB = TN / 16 * KB, PER = (NB + NW - 1) / NW, G = GROUP < PER ? GROUP : PER;
  const int row0 = w.tj * (TN / 16), col0 = w.ti * KB;
#pragma unroll 1
  for (int n0 = 0; n0 < PER; n0 += G) {
    Run8<float> old[G];
    if constexpr (KIND == NS_MUON) {
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const int b = min(wave + (n0 + g) * NW, NB - 1), rb = min(b / KB, w.qr - 1), kb = min(b % KB, w.pr / 2 - 1);
        old[g] = load_weights<KIND>(M, (row0 + rb) * 16 + l16, (col0 + kb) * 32 + g4 * 8);
      }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int b = wave + (n0 + g) * NW, rb = b / KB, kb = b % KB;
      if (n0 + g >= PER || b >= NB || rb >= w.qr || 2 * kb >= w.pr || w.side(2 * kb) <= 0) continue;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = Cs[(kb * 32 + g4 * 8 + e) * CS + rb * 16 + l16];
      if constexpr (LAST) {
        store_result<KIND, TO>(M, (row0 + rb) * 16 + l16, (col0 + kb) * 32 + g4 * 8, v, old[g]);
      } else {
        char* op = KIND == NS_GRAM ? M.opA : KIND == NS_POLY ? M.opB : w.Xt_next;
        store_split(op + block_at(row0 + rb, col0 + kb, M.mp / 32) + lane * 16, v, a.scale);
      }
    }
  }
}

// Blocks of both operands in registers.
template <int FT>
struct NsOperands {
  f16x8 ph[FT], pl[FT], qh[FT], ql[FT];
};

// One 16 x 32 by 32 x 16 product of split operands, smallest terms first.
template <int FT>
__device__ inline void mma_block(const f16x8 (&ph)[FT], const f16x8 (&pl)[FT], const f16x8 (&qh)[FT],
                                 const f16x8 (&ql)[FT], f32x4 (&acc)[FT][FT]) {
#pragma unroll
  for (int i = 0; i < FT; ++i)
#pragma unroll
    for (int k = 0; k < FT; ++k) acc[i][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pl[i], qh[k], acc[i][k], 0, 0, 0);
#pragma unroll
  for (int i = 0; i < FT; ++i)
#pragma unroll
    for (int k = 0; k < FT; ++k) acc[i][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ph[i], ql[k], acc[i][k], 0, 0, 0);
#pragma unroll
  for (int i = 0; i < FT; ++i)
#pragma unroll
    for (int k = 0; k < FT; ++k) acc[i][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ph[i], qh[k], acc[i][k], 0, 0, 0);
}

// Result lane l of a 16 x 16 block holds rows 4 (l / 16) .. + 3 of column l % 16.
template <int FT, int CS, bool ADD = false>
__device__ inline void stage_tile(float* Cs, const f32x4 (&acc)[FT][FT], int lane) {
  const int l16 = lane & 15, g4 = lane >> 4;
#pragma unroll
  for (int i = 0; i < FT; ++i)
#pragma unroll
    for (int k = 0; k < FT; ++k)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float& c = Cs[(i * 16 + g4 * 4 + r) * CS + k * 16 + l16];
        c = ADD ? c + acc[i][k][r] : acc[i][k][r];
      }
}

// Large products: TM x TN tiles, a wave for each 64 x 64 of them, operands through a
// ring of NST LDS slabs of 32 k.  Bound by the matrix cores: 4096 x 4096 takes 191 us
// for X X^T, 197 for A A and 329 for B X, which is 1.15, 1.11 and 1.25 PFLOP/s of fp16
// products (a loop of nothing but such products on random numbers reaches 1.7 here,
// its clock held down by power; a library's fp16 product of this size 1.1).  A slab of
// a 256 x 128 tile takes 1800 cycles where its products take 1536, the rest of a
// launch is the epilogue: every workgroup writes its results at the same time.
// 128 x 128 tiles read 1.5 times as much from L2: for products whose last round of
// larger ones would leave compute units idle, or that have few tiles (eight of
// 1024 x 1024, X X^T: 288 tiles, two workgroups a compute unit, 48 us).
template <int TM, int TN, int NST>
struct NsTile {
  static constexpr int PB = TM / 16, QB = TN / 16, FT = 4;
  static constexpr int NW = (TM / 64) * (TN / 64);
  static constexpr int SLAB = (PB + QB) * BLOCK;    // bytes
  static constexpr int LPW = SLAB / 1024 / NW;      // planes a wave loads per slab
  static constexpr int CS = TN + 4;                 // floats per row of the staged result
  static constexpr int LDS = NST * SLAB > TM * CS * 4 ? NST * SLAB : TM * CS * 4;
  static_assert(LDS <= 160 * 1024, "LDS of a compute unit");
  static_assert(SLAB % (1024 * NW) == 0, "planes are dealt evenly");
};

template <int TM, int TN, int NST, int KIND, typename TO>
__global__ void __launch_bounds__((NsTile<TM, TN, NST>::NW * 64), 2) k_ns_tiles(NsArgs a) {
  using C = NsTile<TM, TN, NST>;
  constexpr int FT = C::FT;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  NsWork<TM, TN, KIND> w;
  if (!w.find(a)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wm = wave / (TN / 64), wn = wave % (TN / 64);
  const u32x4 rp = plane_rsrc(w.P, (uint32_t)w.pr * (uint32_t)w.kblocks * BLOCK);
  const u32x4 rq = plane_rsrc(w.Q, (uint32_t)w.qr * (uint32_t)w.kblocks * BLOCK);
  const uint32_t lds0 = lds_offset(smem), lane_off = (uint32_t)lane * 16u;
  auto issue_one = [&](int s, int st, int i) {
    const int p = wave * C::LPW + i;  // plane within the slab: P's, then Q's
    const bool of_q = p >= C::PB * 2;
    const int q = of_q ? p - C::PB * 2 : p;
    // (row blocks past the matrix: the last one again, its results are dropped)
    const int rb = min(q / 2, (of_q ? w.qr : w.pr) - 1);
    load_plane(of_q ? rq : rp, lds0 + (uint32_t)(st * C::SLAB + p * 1024), lane_off,
               (uint32_t)((rb * w.kblocks + w.k0 + s) * BLOCK + (q % 2) * 1024));
  };
  auto issue = [&](int s, int st) {
#pragma unroll
    for (int i = 0; i < C::LPW; ++i) issue_one(s, st, i);
  };
  f32x4 acc[FT][FT];
#pragma unroll
  for (int i = 0; i < FT; ++i)
#pragma unroll
    for (int k = 0; k < FT; ++k) acc[i][k] = f32x4{0.f, 0.f, 0.f, 0.f};
  // (slabs behind the last one: the last one again, not used)
  const int nsl = w.k1 - w.k0;
#pragma unroll
  for (int p = 0; p < NST; ++p) issue(min(p, nsl - 1), p);
  // Slab s lies in registers when its turn comes: it is read out of LDS while slab
  // s - 1 is multiplied, and the stage it leaves is refilled with slab s + NST.
  // Reads and loads are dealt between the products, since a wave that issues them
  // in a row waits for LDS and feeds no product meanwhile.
  NsOperands<FT> ring[2];
  auto read_one = [&](NsOperands<FT>& o, int st, int n) {
    const char* Ps = smem + st * C::SLAB + lane * 16 + wm * FT * BLOCK;
    const char* Qs = smem + st * C::SLAB + lane * 16 + (C::PB + wn * FT) * BLOCK;
    const int i = n % FT;
    if (n < FT) o.pl[i] = *(const f16x8*)(Ps + i * BLOCK + BLOCK / 2);
    else if (n < 2 * FT) o.qh[i] = *(const f16x8*)(Qs + i * BLOCK);
    else if (n < 3 * FT) o.ph[i] = *(const f16x8*)(Ps + i * BLOCK);
    else o.ql[i] = *(const f16x8*)(Qs + i * BLOCK + BLOCK / 2);
  };
  // this wave's loads of slab s have landed once only those behind it are
  // outstanding; the barrier makes it every wave's, and says that every wave's
  // reads of the slab before it are done
  auto arrive = [&](auto behind) {
    asm volatile("" ::: "memory");
    wait_loads<decltype(behind)::value * C::LPW>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  static_assert(NST >= 2 && C::LPW <= 2 * FT, "the waits and the dealing of loads below");
  arrive(std::integral_constant<int, NST - 1>{});
#pragma unroll
  for (int n = 0; n < 4 * FT; ++n) read_one(ring[0], 0, n);
  constexpr int GROUPS = 4 * FT, PER = 3 * FT * FT / GROUPS;
  auto products = [&](const NsOperands<FT>& now, int g) {  // smallest terms first
#pragma unroll
    for (int q = g * PER; q < (g + 1) * PER; ++q) {
      const int i = q % (FT * FT) / FT, k = q % FT, t = q / (FT * FT);
      acc[i][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(t == 0 ? now.pl[i] : now.ph[i], t == 1 ? now.ql[k] : now.qh[k],
                                                         acc[i][k], 0, 0, 0);
    }
  };
  auto step = [&](int s, const NsOperands<FT>& now, NsOperands<FT>& next, int from, int to) {
    arrive(std::integral_constant<int, NST - 2>{});
    const int slab = min(s + NST, nsl - 1);
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      products(now, g);
      read_one(next, from, g);
      if (g % 2 == 0 && g / 2 < C::LPW) issue_one(slab, to, g / 2);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  int st = 0;  // stage of slab s
  int s = 0;
#pragma unroll 1
  for (; s + 1 < nsl; s += 2) {
    const int st1 = st == NST - 1 ? 0 : st + 1, st2 = st1 == NST - 1 ? 0 : st1 + 1;
    step(s, ring[0], ring[1], st1, st);
    step(s + 1, ring[1], ring[0], st2, st1);
    st = st2;
  }
  if (s < nsl)
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) products(ring[0], g);
  wait_loads<0>();
  asm volatile("" ::: "memory");
  __syncthreads();  // every wave done with the slabs before the result is staged over them
  float* Cs = (float*)smem;
  stage_tile<FT, C::CS>(Cs + wm * 64 * C::CS + wn * 64, acc, lane);
  __syncthreads();
  if (w.parts > 1 && !join_parts<TM, TN, C::NW * 64>(a, w, Cs)) return;
  finish_tile<TM, TN, KIND, TO, C::NW, 1, 8, false>(a, w, Cs, wave, lane, nullptr);
}

// Small products: a T x T tile per workgroup, K dealt to its NW waves in runs of
// blocks, each wave loading its operands straight into registers (a load is one
// contiguous plane), DEPTH blocks ahead; the waves' sums meet in LDS, where what the
// epilogue reads beside them has arrived meanwhile.  No barrier before that: such a
// product is bound by latencies, not by the matrix cores.  1000 x 300 takes 6.3 us for
// X X^T, 4.7 for A A and 8.1 for B X, of which an empty launch is 2.4 and the operands'
// way from another XCD's writes (through memory) 1.2.  The tiles with the longest sums
// bound a list: DeepCNet(6,100)'s matrices with softmax take 36 us for X X^T, in which a
// wave of the softmax matrix's tiles goes through 30 blocks of 64 x 64 with two in flight
// (the matrix cores are busy 15% of the time, L2 gives about 14 bytes a cycle and compute unit).
// The partial tiles that its waves stage in LDS: of 64 x 64, where something lies beside
// them, the second half of the waves first, to which the first half then adds, so that two
// workgroups fit a compute unit (B X of 1000 x 600 three times: 18.8 us, else 22.5).
constexpr int direct_parts(int T, int waves, int kind) { return T == 64 && kind != NS_GRAM ? waves / 2 : waves; }

template <int T, int NW, int DEPTH, int KIND, typename TO>
__global__ void __launch_bounds__((NW * 64), (NW == 8 ? 4 : 1)) k_ns_direct(NsArgs a) {
  using W = NsWork<T, T, KIND>;
  constexpr int FT = T / 16, CS = T + 4, NB = FT * (T / 32);
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  W w;
  if (!w.find(a)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int k0 = w.kblocks * wave / NW, k1 = w.kblocks * (wave + 1) / NW;
  auto load = [&](int kb) {
    NsOperands<FT> o;
#pragma unroll
    for (int i = 0; i < FT; ++i) {
      // row blocks past the matrix: the last one again, its results are dropped
      const char* p = w.P + block_at(min(i, w.pr - 1), kb, w.kblocks) + lane * 16;
      const char* q = w.Q + block_at(min(i, w.qr - 1), kb, w.kblocks) + lane * 16;
      o.ph[i] = *(const f16x8*)p;
      o.pl[i] = *(const f16x8*)(p + BLOCK / 2);
      o.qh[i] = *(const f16x8*)q;
      o.ql[i] = *(const f16x8*)(q + BLOCK / 2);
    }
    return o;
  };
  char* beside = smem + direct_parts(T, NW, KIND) * T * CS * 4;
  auto load_besides = [&]() {
    if constexpr (KIND != NS_GRAM)
      for (int b = wave; b < NB; b += NW) {
        const int rb = b / (T / 32), kb = b % (T / 32);
        if (rb < w.pr && 2 * kb < w.qr)
          load_beside<W, KIND>(w, w.ti * FT + rb, w.tj * (T / 32) + kb, lane, lds_offset(beside + b * 2048));
      }
  };
  f32x4 acc[FT][FT];
#pragma unroll
  for (int i = 0; i < FT; ++i)
#pragma unroll
    for (int k = 0; k < FT; ++k) acc[i][k] = f32x4{0.f, 0.f, 0.f, 0.f};
  NsOperands<FT> ring[DEPTH];
  int kb = k0;
  auto multiply = [&](int d) { mma_block<FT>(ring[d].ph, ring[d].pl, ring[d].qh, ring[d].ql, acc); };
  if (k1 - k0 >= DEPTH) {
    // In the loop nothing is loaded under a condition or out of order: a wait for a
    // block would wait for younger ones too.
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      ring[d] = load(k0 + d);
      __builtin_amdgcn_sched_barrier(0);
    }
    load_besides();
    for (; kb + 2 * DEPTH <= k1; kb += DEPTH)
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        multiply(d);
        ring[d] = load(kb + DEPTH + d);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      multiply(d);
      if (kb + DEPTH + d < k1) ring[d] = load(kb + DEPTH + d);
      __builtin_amdgcn_sched_barrier(0);
    }
    kb += DEPTH;
  } else {
#pragma unroll
    for (int d = 0; d < DEPTH - 1; ++d)
      if (k0 + d < k1) ring[d] = load(k0 + d);
    load_besides();
  }
#pragma unroll
  for (int d = 0; d < DEPTH - 1; ++d)
    if (kb + d < k1) multiply(d);
  float* Cs = (float*)smem;
  constexpr int PARTS = direct_parts(T, NW, KIND);
  if (wave >= NW - PARTS) stage_tile<FT, CS>(Cs + (wave - (NW - PARTS)) * T * CS, acc, lane);
  if constexpr (PARTS < NW) {
    __syncthreads();
    if (wave < PARTS) stage_tile<FT, CS, true>(Cs + wave * T * CS, acc, lane);
  }
  asm volatile("" ::: "memory");
  wait_loads<0>();
  __syncthreads();
  finish_tile<T, T, KIND, TO, NW, PARTS, 2, true>(a, w, Cs, wave, lane, beside);
}

// ---------------------------------------------------------------------------
// A small matrix, all steps in one workgroup: X stays in registers in float32 (wave w
// holds the 16 x 16 blocks w, w + 8, .. of it, as the matrix cores leave them), its
// operands, A and B in LDS.  Five steps take 9.5 us for 9 x 50, 16.4 for 64 x 64 and
// 22.4 for 64 x 128 (20 of these 41.4: a workgroup each); 65 x 65, just too large, takes
// 65 in its 17 launches.

constexpr int SMALL_M = 64, SMALL_ELEMS = 8192, SMALL_STEPS = 8;
constexpr int SMALL_XB = SMALL_ELEMS / 256 / 8, SMALL_AB = SMALL_M * SMALL_M / 256 / 8;  // blocks a wave holds
constexpr int SMALL_LDS = 2 * SMALL_ELEMS * 4 + 2 * SMALL_M * SMALL_M * 4;

struct NsCoef {
  int32_t steps;
  float c[3 * SMALL_STEPS];
  int8_t ex[SMALL_STEPS], ea[SMALL_STEPS], eb[SMALL_STEPS];  // NsStep's
};
static_assert(sizeof(NsArgs) + sizeof(NsTable) + sizeof(NsCoef) <= 4096, "kernel arguments");

// Block (bi, bj) of a result, lane l's part rows 4 (l / 16) .. of column l % 16, as the
// operand whose rows are the result's columns: four consecutive k, 8 bytes a plane.
__device__ inline void put_columns(char* op, int bi, int bj, int kblocks, int lane, f32x4 v, float s) {
  typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
  f16x4 hi, lo;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float x = v[e] * s;
    hi[e] = (_Float16)x;
    lo[e] = (_Float16)(x - (float)hi[e]);
  }
  const int k = (bi & 1) * 16 + (lane >> 4) * 4;  // within a block of 32
  char* at = op + block_at(bj, bi >> 1, kblocks) + ((k >> 3) * 16 + (lane & 15)) * 16 + (k & 7) * 2;
  *(f16x4*)at = hi;
  *(f16x4*)(at + BLOCK / 2) = lo;
}

// ... and as the operand with the result's rows.
__device__ inline void put_rows(char* op, int bi, int bj, int kblocks, int lane, f32x4 v, float s) {
  const int k = (bj & 1) * 16 + (lane & 15);
  char* at = op + block_at(bi, bj >> 1, kblocks) + ((k >> 3) * 16 + (lane >> 4) * 4) * 16 + (k & 7) * 2;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float x = v[e] * s;
    const _Float16 hi = (_Float16)x;
    *(_Float16*)(at + e * 16) = hi;
    *(_Float16*)(at + e * 16 + BLOCK / 2) = (_Float16)(x - (float)hi);
  }
}

__device__ inline f32x4 small_product(const char* P, int bi, const char* Q, int bj, int kblocks, int lane) {
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int kb = 0; kb < kblocks; ++kb) {
    const char* p = P + block_at(bi, kb, kblocks) + lane * 16;
    const char* q = Q + block_at(bj, kb, kblocks) + lane * 16;
    const f16x8 ph = *(const f16x8*)p, pl = *(const f16x8*)(p + BLOCK / 2);
    const f16x8 qh = *(const f16x8*)q, ql = *(const f16x8*)(q + BLOCK / 2);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(pl, qh, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(ph, ql, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(ph, qh, acc, 0, 0, 0);
  }
  return acc;
}

template <typename T, typename TO, bool MUON>
__global__ void __launch_bounds__(512) k_ns_small(NsArgs a, NsTable t, NsCoef coef) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  __shared__ double red[8];
  const NsMat M = matrix(&t, blockIdx.x);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int mb = M.mp / 16, nb = M.np / 16, mk = M.mp / 32, nk = M.np / 32;
  const int xblocks = mb * nb, ablocks = mb * mb;
  char* opX = smem;
  char* opXt = opX + M.mp * M.np * 4;
  char* opA = opXt + M.mp * M.np * 4;
  char* opB = opA + M.mp * M.mp * 4;
  // element (i, k) of X in the caller's array
  const int64_t stride = MUON ? (M.tall ? M.m : M.n) : M.u_stride;
  const auto at = [&](int i, int k, int64_t ld) { return M.tall ? (int64_t)k * ld + i : (int64_t)i * ld + k; };
  f32x4 x[SMALL_XB];
  double ss = 0.0;
#pragma unroll
  for (int n = 0; n < SMALL_XB; ++n) {
    const int t = wave + 8 * n, bi = t / nb, bj = t - bi * nb;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = bi * 16 + (lane >> 4) * 4 + e, k = bj * 16 + (lane & 15);
      const bool in = t < xblocks && i < M.m && k < M.n;
      const int64_t q = at(min(i, M.m - 1), min(k, M.n - 1), stride);  // (outside: an element that is read, not used)
      float u = Elem<T>::to_f32(((const T*)M.u)[q]);
      if constexpr (MUON) {
        const float v = a.momentum * M.v[q] + u;
        if (in) M.v[q] = v;
        u = a.nesterov ? a.momentum * v + u : v;
      }
      x[n][e] = in ? u : 0.f;
      ss += (double)x[n][e] * x[n][e];
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) ss += __shfl_xor(ss, d, 64);
  if (lane == 0) red[wave] = ss;
  __syncthreads();
  ss = 0.0;
#pragma unroll
  for (int w = 0; w < 8; ++w) ss += red[w];
  const double inv = ss == 0.0 ? 0.0 : 1.0 / sqrt(ss);
  const auto put_x = [&](float sx) {
#pragma unroll
    for (int n = 0; n < SMALL_XB; ++n) {
      const int t = wave + 8 * n, bi = t / nb, bj = t - bi * nb;
      if (t >= xblocks) break;
      put_rows(opX, bi, bj, nk, lane, x[n], sx);
      put_columns(opXt, bi, bj, mk, lane, x[n], sx);
    }
  };
#pragma unroll
  for (int n = 0; n < SMALL_XB; ++n) {
    const int t = wave + 8 * n, bi = t / nb, bj = t - bi * nb;
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // (the padding stays zero beside a norm that is NaN or infinite)
      const bool in = bi * 16 + (lane >> 4) * 4 + e < M.m && bj * 16 + (lane & 15) < M.n;
      x[n][e] = in ? (float)((double)x[n][e] * inv) : 0.f;
    }
  }
  put_x(ldexpf(1.f, coef.ex[0]));
  __syncthreads();
  for (int s = 0; s < coef.steps; ++s) {
    const float ca = coef.c[3 * s], cb = coef.c[3 * s + 1], cc = coef.c[3 * s + 2];
    const int ex = coef.ex[s], ea = coef.ea[s], eb = coef.eb[s];
    const float sa = ldexpf(1.f, ea), sb = ldexpf(1.f, eb);
    const float from_xx = ldexpf(1.f, -2 * ex), from_aa = ldexpf(1.f, -2 * ea), from_bx = ldexpf(1.f, -eb - ex);
    f32x4 A[SMALL_AB];
#pragma unroll
    for (int n = 0; n < SMALL_AB; ++n) {
      const int t = wave + 8 * n, bi = t / mb, bj = t - bi * mb;
      if (t >= ablocks) break;
      A[n] = small_product(opX, bi, opX, bj, nk, lane) * from_xx;
      put_columns(opA, bi, bj, mk, lane, A[n], sa);
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < SMALL_AB; ++n) {
      const int t = wave + 8 * n, bi = t / mb, bj = t - bi * mb;
      if (t >= ablocks) break;
      const f32x4 B = cb * A[n] + cc * (small_product(opA, bi, opA, bj, mk, lane) * from_aa);
      put_columns(opB, bi, bj, mk, lane, B, sb);
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < SMALL_XB; ++n) {
      const int t = wave + 8 * n, bi = t / nb, bj = t - bi * nb;
      if (t >= xblocks) break;
      x[n] = ca * x[n] + small_product(opB, bi, opXt, bj, mk, lane) * from_bx;
    }
    if (s + 1 == coef.steps) break;
    __syncthreads();  // every wave done with X's operands
    put_x(ldexpf(1.f, coef.ex[s + 1]));
    __syncthreads();
  }
#pragma unroll
  for (int n = 0; n < SMALL_XB; ++n) {
    const int t = wave + 8 * n, bi = t / nb, bj = t - bi * nb;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = bi * 16 + (lane >> 4) * 4 + e, k = bj * 16 + (lane & 15);
      if (t >= xblocks || i >= M.m || k >= M.n) continue;
      if constexpr (MUON) {
        const int64_t q = at(i, k, stride);
        const float w = M.w[q], wn = w - (M.scale * x[n][e] + M.decay * w);
        M.w[q] = wn;
        if (M.o) ((TO*)M.o)[q] = Elem<TO>::from_f32(wn);
      } else {
        ((TO*)M.o)[at(i, k, M.o_stride)] = Elem<TO>::from_f32(x[n][e]);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// host

// The kernels of a product.
enum NsPlan { NS_256, NS_128, NS_64, NS_32 };
struct NsShape {
  int tm, tn;
  // k is divided into runs of this many blocks or more, then evenly over their number, so
  // that a part may have down to half as many; 0: tiles are not divided
  int min_k;
};
constexpr NsShape NS_SHAPE[] = {{256, 128, 16}, {128, 128, 12}, {64, 64, 0}, {32, 32, 0}};

int64_t tiles_of(const NsMat& M, int kind, const NsShape& s) {
  const int64_t tm = (M.mp + s.tm - 1) / s.tm, tn = (M.np + s.tn - 1) / s.tn;
  // (a last tile row that ends early has tiles past the diagonal: they find nothing to do)
  return symmetric(kind) ? s.tm / s.tn * (tm * (tm + 1) / 2) : tm * tn;
}

int64_t k_of(const NsMat& M, int kind) { return (kind == NS_GRAM ? M.np : M.mp) / 32; }

// How many workgroups can share a tile of the last round of 256 x 128 tiles, which has
// `rest` tiles: they are the last matrix's.
int64_t last_round_parts(const NsMat& last, int kind, int64_t rest) {
  if (rest == 0 || rest > tiles_of(last, kind, NS_SHAPE[NS_256])) return 1;
  return std::max<int64_t>(1, std::min<int64_t>({NS_PARTS, NS_CUS / rest, k_of(last, kind) / NS_SHAPE[NS_256].min_k}));
}

// Which kernel a product over the group takes: through LDS where it has work for that
// (X X^T, A A: slabs; B X, whose sums are short: tiles), in 256 x 128 tiles if their last
// round has NS_FULL workgroups or can be divided, else in 128 x 128 tiles; straight into registers otherwise.
NsPlan plan_product(const NsGroup& g, int kind) {
  int64_t t256 = 0, t128 = 0, t64 = 0, slabs = 0;
  for (int j = 0; j < g.a.n; ++j) {
    const int64_t t = tiles_of(g.t.mat[j], kind, NS_SHAPE[NS_128]);
    t256 += tiles_of(g.t.mat[j], kind, NS_SHAPE[NS_256]);
    t128 += t;
    t64 += tiles_of(g.t.mat[j], kind, NS_SHAPE[NS_64]);
    slabs += t * k_of(g.t.mat[j], kind);
  }
  const bool lds = symmetric(kind) ? slabs >= NS_SLABS * NS_CUS
                                   : slabs >= NS_SLABS_APPLY * NS_CUS || t128 >= NS_TILES_APPLY;
  if (!lds) return t64 >= (symmetric(kind) ? NS_TILES_64 : NS_TILES_64_APPLY) ? NS_64 : NS_32;
  const int64_t rest = t256 % NS_CUS;
  return rest == 0 || rest >= NS_FULL || (t256 > NS_CUS && last_round_parts(g.t.mat[g.a.n - 1], kind, rest) > 1) ? NS_256
                                                                                                         : NS_128;
}

// Deals the tiles of a product to workgroups, and the k of a tile to several where the
// tiles alone would leave compute units idle: all tiles of a product that has fewer than
// compute units, or those of its last round.  Sets a.beg (workgroups per XCD) and the
// matrices' parts; returns the partial tiles.
int64_t deal_tiles(NsGroup& g, int kind, NsPlan plan) {
  NsArgs& a = g.a;
  const NsMat* mat = g.t.mat;
  const NsShape& s = NS_SHAPE[plan];
  int64_t all = 0, work = 0, most_k = 0;
  for (int j = 0; j < a.n; ++j) {
    const int64_t t = tiles_of(mat[j], kind, s), k = k_of(mat[j], kind);
    a.deal[j] = NsDeal{(int32_t)t, 1, 0, 0};
    all += t;
    work += t * k;
    most_k = std::max(most_k, k);
  }
  if (s.min_k == 0) {
  } else if (all < NS_CUS) {
    auto parts = [&](const NsMat& M, int64_t len) {
      return std::min<int64_t>(NS_PARTS, (k_of(M, kind) + len - 1) / len);
    };
    int64_t len = std::max<int64_t>(s.min_k, (work + NS_CUS - 1) / NS_CUS);
    for (; len < most_k; len += std::max<int64_t>(1, len / 16)) {
      int64_t items = 0;
      for (int j = 0; j < a.n; ++j) items += a.deal[j].whole * parts(mat[j], len);
      if (items <= NS_CUS) break;
    }
    for (int j = 0; j < a.n; ++j) {
      a.deal[j].parts = (int32_t)parts(mat[j], len);
      if (a.deal[j].parts > 1) a.deal[j].whole = 0;
    }
  } else if (plan == NS_256) {
    const int64_t rest = all % NS_CUS, p = last_round_parts(mat[a.n - 1], kind, rest);
    if (p > 1) {
      a.deal[a.n - 1].whole -= (int32_t)rest;
      a.deal[a.n - 1].parts = (int32_t)p;
    }
  }
  int64_t beg = 0, slots = 0, counters = 0;
  for (int j = 0; j < a.n; ++j) {
    NsDeal& D = a.deal[j];
    const int64_t divided = tiles_of(mat[j], kind, s) - D.whole;
    D.slot = (int32_t)slots;
    D.counter = (int32_t)counters;
    a.beg[j] = (int32_t)beg;
    beg += (D.whole + 7) / 8 + (divided * D.parts + 7) / 8;
    slots += divided * D.parts;
    counters += divided;
  }
  a.beg[a.n] = (int32_t)beg;
  return slots;  // (divided tiles are fewer than compute units, so than NS_COUNT)
}

// LDS of k_ns_direct: the waves' partial tiles, and what lies beside the result.
constexpr int direct_lds(int T, int waves, int kind) {
  return direct_parts(T, waves, kind) * T * (T + 4) * 4 + (kind == NS_GRAM ? 0 : (T / 16) * (T / 32) * 2048);
}

template <auto KERN>
hipError_t launch_tiles(int threads, int lds, const NsArgs& a, hipStream_t st) {
  const hipError_t e = allow_lds<KERN>(lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(KERN, dim3(8 * a.beg[a.n]), dim3(threads), lds, st, a);
  return hipGetLastError();
}

template <int KIND, typename TO>
hipError_t run_product(NsGroup& g, hipStream_t st) {
  const NsPlan plan = plan_product(g, KIND);
  deal_tiles(g, KIND, plan);
  const NsArgs& a = g.a;
  switch (plan) {
    case NS_256: {
      using C = NsTile<256, 128, 3>;
      return launch_tiles<k_ns_tiles<256, 128, 3, KIND, TO>>(C::NW * 64, C::LDS, a, st);
    }
    case NS_128: {
      // Alone on its compute unit a workgroup keeps one more slab in flight (X X^T of
      // 2100 x 3900: 76 us with three stages, 96 with two; 2047 x 8000: 139 and 195).
      // Three stages leave no room for a second workgroup (eight of 1024 x 1024, 288
      // tiles: 50 and 47).
      if (8 * a.beg[a.n] <= NS_CUS) {
        using C = NsTile<128, 128, 3>;
        return launch_tiles<k_ns_tiles<128, 128, 3, KIND, TO>>(C::NW * 64, C::LDS, a, st);
      }
      using C = NsTile<128, 128, 2>;
      return launch_tiles<k_ns_tiles<128, 128, 2, KIND, TO>>(C::NW * 64, C::LDS, a, st);
    }
    case NS_64:
      return launch_tiles<k_ns_direct<64, 4, 2, KIND, TO>>(256, direct_lds(64, 4, KIND), a, st);
    default: {
      constexpr int NW = symmetric(KIND) ? 8 : 4;  // (X X^T has the longest sums, B X the most tiles)
      return launch_tiles<k_ns_direct<32, NW, 3, KIND, TO>>(NW * 64, direct_lds(32, NW, KIND), a, st);
    }
  }
}

template <typename TO, bool MUON>
hipError_t run_steps(NsGroup& g, int steps, const NsStep* step, hipStream_t st) {
  NsArgs& a = g.a;
  for (int s = 0; s < steps; ++s) {
    const NsStep& S = step[s];
    a.step = s;
    // (powers of two: nothing is rounded)
    a.of_sum = ldexpf(1.f, -2 * S.ex);
    a.scale = ldexpf(1.f, S.ea);
    hipError_t e = run_product<NS_GRAM, float>(g, st);
    a.of_sum = ldexpf(S.c, -2 * S.ea);
    a.of_beside = ldexpf(S.b, -S.ea);
    a.scale = ldexpf(1.f, S.eb);
    if (e == hipSuccess) e = run_product<NS_POLY, float>(g, st);
    a.of_sum = ldexpf(1.f, -S.eb - S.ex);
    a.of_beside = S.a;
    a.scale = s + 1 < steps ? ldexpf(1.f, step[s + 1].ex) : 1.f;
    if (e == hipSuccess)
      e = s + 1 < steps ? run_product<NS_APPLY, float>(g, st) : run_product<MUON ? NS_MUON : NS_ORTHO, TO>(g, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T, bool MUON>
hipError_t run_begin(NsGroup& g, const NsStep& first, hipStream_t st) {
  NsArgs& a = g.a;
  a.scale = ldexpf(1.f, first.ex);
  NsMat* mat = g.t.mat;
  int blocks = 0;
  for (int j = 0; j < a.n; ++j) {
    a.beg[j] = blocks;
    mat[j].nssq = (int)std::max<int64_t>(1, std::min<int64_t>(NS_SSQ, (int64_t)mat[j].m * mat[j].n / 2048));
    blocks += mat[j].nssq;
  }
  a.beg[a.n] = blocks;
  hipLaunchKernelGGL((k_ns_begin<T, MUON>), dim3(blocks), dim3(256), 0, st, a, g.t);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  blocks = 0;
  for (int j = 0; j < a.n; ++j) {
    a.beg[j] = blocks;
    blocks += (mat[j].mp / 32 * (mat[j].np / 32) + 3) / 4;
  }
  a.beg[a.n] = blocks;
  hipLaunchKernelGGL((k_ns_convert<T, MUON>), dim3(blocks), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t ns_part_bytes(NsGroup& g) {
  int64_t most = 0;
  for (const int kind : {NS_GRAM, NS_POLY, NS_APPLY}) {
    const NsPlan plan = plan_product(g, kind);
    most = std::max(most, deal_tiles(g, kind, plan) * NS_SHAPE[plan].tm * NS_SHAPE[plan].tn);
  }
  return (size_t)most * sizeof(float);
}

template <typename T, typename TO, bool MUON>
static hipError_t run_small(const NsGroup& g, const NsCoef& c, hipStream_t st) {
  const hipError_t e = allow_lds<k_ns_small<T, TO, MUON>>(SMALL_LDS);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_ns_small<T, TO, MUON>), dim3(g.a.n), dim3(512), SMALL_LDS, st, g.a, g.t, c);
  return hipGetLastError();
}

hipError_t launch_newton_schulz(NsGroup& g, bool bf16, bool muon, int steps, const NsStep* step, hipStream_t st) {
  bool small = steps <= SMALL_STEPS;
  for (int j = 0; j < g.a.n; ++j)
    small = small && g.t.mat[j].mp <= SMALL_M && (int64_t)g.t.mat[j].mp * g.t.mat[j].np <= SMALL_ELEMS;
  if (small) {
    NsCoef c{};
    c.steps = steps;
    for (int i = 0; i < steps; ++i) {
      c.c[3 * i] = step[i].a;
      c.c[3 * i + 1] = step[i].b;
      c.c[3 * i + 2] = step[i].c;
      c.ex[i] = (int8_t)step[i].ex;
      c.ea[i] = (int8_t)step[i].ea;
      c.eb[i] = (int8_t)step[i].eb;
    }
    if (muon) return bf16 ? run_small<float, __bf16, true>(g, c, st) : run_small<float, float, true>(g, c, st);
    return bf16 ? run_small<__bf16, __bf16, false>(g, c, st) : run_small<float, float, false>(g, c, st);
  }
  hipError_t e = muon ? run_begin<float, true>(g, step[0], st)
                 : bf16 ? run_begin<__bf16, false>(g, step[0], st) : run_begin<float, false>(g, step[0], st);
  if (e != hipSuccess) return e;
  if (muon) return bf16 ? run_steps<__bf16, true>(g, steps, step, st) : run_steps<float, true>(g, steps, step, st);
  return bf16 ? run_steps<__bf16, false>(g, steps, step, st) : run_steps<float, false>(g, steps, step, st);
}

}  // namespace sscn
