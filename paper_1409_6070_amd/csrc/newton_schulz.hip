// Orthogonalising matrices by Newton-Schulz products, and the weight update that
// uses the result (Muon).
//
//   X = u / |u|_F  (m x n with m <= n: transposed where u is taller than wide)
//   each step:  A = X X^T,  B = b A + c A A,  X <- a X + B X
//
// The odd polynomial p(s) = a s + b s^3 + c s^5 acts on X's singular values and
// leaves its singular vectors: a few steps bring all but the smallest near 1.
//
// Precision.  X is kept in float32.  A product's operands are split into two
// fp16 numbers each, hi + lo (22 bits; powers of two keep them in fp16's range),
// and multiplied on the fp16 matrix cores as hi hi + hi lo + lo hi with float32
// sums: three times the matrix work of a plain fp16 product, and still a fifth of
// the time of float32 MFMA.  A small singular value is carried from step to step
// by a X alone (B's rows along it are small), which is float32 throughout: the
// result is as near to the formula's as a float32 computation's, where operands
// of fewer bits lose the small singular values, whose errors every step
// multiplies by a (about 3.4).
//
// Layout.  An operand with R rows of K values is stored as the matrix cores read
// it: blocks of 16 rows x 32 k, row-block major, a block's hi plane of 1 KiB then
// its lo plane, lane l's 16 bytes being row l % 16, k 8 (l / 16) .. + 7.  One wave
// moves a plane with one 16-byte load per lane straight into LDS and reads it
// back the same way: contiguous everywhere, no bank conflicts, no swizzle.  Rows
// and columns are padded with zeros to the tile edge, so no product checks bounds.

#include "common.h"
#include "kernels.h"

namespace sscn {

static_assert(sizeof(NsArgs) <= 4096, "kernel arguments must fit the 4 KiB argument segment");

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Powers of two that the planes carry.  The entry points admit coefficients that
// keep X's singular values at most 3.5, so entries of A at most 12.25, and those of
// B at most 200: all below fp16's 65504, with lo parts above its smallest steps.
constexpr float SX = 256.f, SA = 4096.f, SB = 256.f;

constexpr int BLOCK = 2048;  // bytes of a 16 x 32 block, both planes

// s_waitcnt vmcnt(n) lgkmcnt(0)
template <int N>
__device__ inline void wait_loads() {
  static_assert(N >= 0 && N < 64, "vmcnt field");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
}

// One 16-byte load per lane into LDS: lane l's bytes land at lds + 16 l.  The
// compiler does not see it; wait_loads and the barriers' fences order it.
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

__device__ inline void load_split(const char* at, float (&v)[8], float inv) {
  const f16x8 hi = *(const f16x8*)at, lo = *(const f16x8*)(at + BLOCK / 2);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = ((float)hi[e] + (float)lo[e]) * inv;
}

// Address of lane l's part of block (rb, kb) of an operand with kblocks blocks a row.
__device__ inline int64_t block_at(int rb, int kb, int kblocks) { return ((int64_t)rb * kblocks + kb) * BLOCK; }

__device__ inline int find_mat(const NsArgs& a, int t) {
  int j = 0;
  while (j + 1 < a.n && t >= a.beg[j + 1]) ++j;
  return j;
}

// ---------------------------------------------------------------------------
// |u|_F^2 as partial sums in float64 (any float32 matrix's fits), and for Muon
// the velocity: v <- mu v + g.  NS_SSQ workgroups at most per matrix.

template <typename T, bool MUON>
__global__ void __launch_bounds__(256) k_ns_begin(NsArgs a) {
  const int j = find_mat(a, blockIdx.x);
  const NsMat& M = a.mat[j];
  const int blk = blockIdx.x - a.beg[j], nblk = a.beg[j + 1] - a.beg[j];
  const int64_t rows = M.tall ? M.n : M.m, cols = M.tall ? M.m : M.n;
  double s = 0.0;
  if constexpr (MUON) {
    const float* g = (const float*)M.u;
    for (int64_t i = (int64_t)blk * 256 + threadIdx.x; i < rows * cols; i += (int64_t)nblk * 256) {
      const float gi = g[i], v = a.momentum * M.v[i] + gi;
      M.v[i] = v;
      const float u = a.nesterov ? a.momentum * v + gi : v;
      s += (double)u * u;
    }
  } else {
    const T* u = (const T*)M.u;
    int tx = 256;  // threads along a row: short rows go several at a time
    while (tx / 2 >= cols) tx /= 2;
    for (int64_t r = (int64_t)blk * (256 / tx) + threadIdx.x / tx; r < rows; r += (int64_t)nblk * (256 / tx))
#pragma unroll 4
      for (int64_t c = threadIdx.x % tx; c < cols; c += tx) {
        const double x = Elem<T>::to_f32(u[r * M.u_stride + c]);
        s += x * x;
      }
  }
  __shared__ double red[256];
  red[threadIdx.x] = s;
  __syncthreads();
  for (int w = 128; w > 0; w >>= 1) {
    if ((int)threadIdx.x < w) red[threadIdx.x] += red[threadIdx.x + w];
    __syncthreads();
  }
  if (threadIdx.x == 0) M.ssq[blk] = red[0];
}

// X = u / |u|_F in float32 and as both operands; a wave per 32 x 32 tile.
template <typename T, bool MUON>
__global__ void __launch_bounds__(256) k_ns_convert(NsArgs a) {
  const int j = find_mat(a, blockIdx.x);
  const NsMat& M = a.mat[j];
  __shared__ double red[256];
  __shared__ float tile[4][32][36];
  double ss = 0.0;
  for (int k = threadIdx.x; k < M.nssq; k += 256) ss += M.ssq[k];
  red[threadIdx.x] = ss;
  __syncthreads();
  for (int w = 128; w > 0; w >>= 1) {
    if ((int)threadIdx.x < w) red[threadIdx.x] += red[threadIdx.x + w];
    __syncthreads();
  }
  const double inv = red[0] == 0.0 ? 0.0 : 1.0 / sqrt(red[0]);  // (a zero matrix stays zero)
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int tn = M.np / 32, t = (blockIdx.x - a.beg[j]) * 4 + wave;
  const bool live = t < (M.mp / 32) * tn;
  const int i0 = t / tn * 32, j0 = t % tn * 32;
  if (live) {
    // lanes along the caller's rows
    const int q = lane & 31;
#pragma unroll 8
    for (int p = lane >> 5; p < 32; p += 2) {
      const int i = i0 + (M.tall ? q : p), c = j0 + (M.tall ? p : q);
      float x = 0.f;
      if (i < M.m && c < M.n) {
        const int64_t r = M.tall ? c : i, k = M.tall ? i : c;
        if constexpr (MUON) {
          const int64_t at = r * (M.tall ? M.m : M.n) + k;
          const float v = M.v[at];
          x = a.nesterov ? a.momentum * v + ((const float*)M.u)[at] : v;
        } else {
          x = Elem<T>::to_f32(((const T*)M.u)[r * M.u_stride + k]);
        }
        x = (float)((double)x * inv);
      }
      tile[wave][i - i0][c - j0] = x;
    }
  }
  __syncthreads();
  if (!live) return;
  const int r16 = lane & 15, k8 = lane >> 4;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float v[8];
    const int i = h * 16 + r16;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = tile[wave][i][k8 * 8 + e];
    float* X = M.X + (int64_t)(i0 + i) * M.np + j0 + k8 * 8;
    *(f32x4*)X = f32x4{v[0], v[1], v[2], v[3]};
    *(f32x4*)(X + 4) = f32x4{v[4], v[5], v[6], v[7]};
    store_split(M.opX + block_at(i0 / 16 + h, j0 / 32, M.np / 32) + lane * 16, v, SX);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = tile[wave][k8 * 8 + e][h * 16 + r16];
    store_split(M.opXt[0] + block_at(j0 / 16 + h, i0 / 32, M.mp / 32) + lane * 16, v, SX);
  }
}

// ---------------------------------------------------------------------------
// the products: C[i][j] = sum_k P[i][k] Q[j][k]

enum NsKind { NS_GRAM, NS_POLY, NS_APPLY, NS_ORTHO, NS_MUON };

// T x T result tiles of four waves (2 x 2), KB blocks of k per slab, NST slabs in LDS.
template <int T, int KB, int NST>
struct NsTile {
  static constexpr int RB = T / 16;                     // row blocks of an operand's tile
  static constexpr int FT = T / 32;                     // 16 x 16 results per wave and side
  static constexpr int SLAB = 2 * RB * KB * BLOCK;      // bytes
  static constexpr int LPW = SLAB / 1024 / 4;           // planes a wave loads per slab
  static constexpr int CS = T + 4;                      // floats per row of the staged result
  static constexpr int LDS = NST * SLAB > T * CS * 4 ? NST * SLAB : T * CS * 4;
  static_assert(SLAB % 4096 == 0, "planes are dealt to four waves");
};

template <int T, int KB, int NST, int KIND, typename TO>
__global__ void __launch_bounds__(256) k_ns_product(NsArgs a) {
  using C = NsTile<T, KB, NST>;
  constexpr int FT = C::FT, RB = C::RB;
  constexpr bool SYM = KIND == NS_GRAM || KIND == NS_POLY;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  // consecutive tiles on one XCD, whose L2 they share
  const int total = a.beg[a.n], per = (total + 7) / 8;
  const int tix = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || tix >= total) return;
  const int j = find_mat(a, tix);
  const NsMat& M = a.mat[j];
  int t = tix - a.beg[j], ti, tj;
  if constexpr (SYM) {  // tiles on and below the diagonal
    ti = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while (ti * (ti + 1) / 2 > t) --ti;
    while ((ti + 1) * (ti + 2) / 2 <= t) ++ti;
    tj = t - ti * (ti + 1) / 2;
  } else {
    ti = t / (M.np / T);
    tj = t - ti * (M.np / T);
  }
  ti = __builtin_amdgcn_readfirstlane(ti);
  tj = __builtin_amdgcn_readfirstlane(tj);
  const int kblocks = (KIND == NS_GRAM ? M.np : M.mp) / 32;
  const char* P = KIND == NS_GRAM ? M.opX : KIND == NS_POLY ? M.opA : M.opB;
  const char* Q = KIND == NS_GRAM ? M.opX : KIND == NS_POLY ? M.opA : M.opXt[a.parity];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wm = wave >> 1, wn = wave & 1;
  const uint32_t span = (uint32_t)RB * (uint32_t)kblocks * BLOCK;  // a row tile of an operand
  const u32x4 rs = wave < 2 ? plane_rsrc(P + (int64_t)ti * span, span) : plane_rsrc(Q + (int64_t)tj * span, span);
  const uint32_t lds0 = lds_offset(smem);
  const uint32_t lane_off = (uint32_t)lane * 16u;
  // waves 0 and 1 load P's planes of a slab, 2 and 3 Q's
  auto issue = [&](int s, int st) {
#pragma unroll
    for (int i = 0; i < C::LPW; ++i) {
      const int p = wave * C::LPW + i;                 // plane within the slab
      const int q = p % (RB * KB * 2);                 // within its operand
      const int rb = q / (KB * 2), rest = q % (KB * 2);  // row block, then (k block, plane): contiguous
      load_plane(rs, lds0 + (uint32_t)(st * C::SLAB + p * 1024), lane_off,
                 (uint32_t)((rb * kblocks + s * KB) * BLOCK + rest * 1024));
    }
  };
  f32x4 acc[FT][FT];
#pragma unroll
  for (int i = 0; i < FT; ++i)
#pragma unroll
    for (int k = 0; k < FT; ++k) acc[i][k] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int nsl = kblocks / KB;
#pragma unroll
  for (int p = 0; p < NST - 1; ++p)
    if (p < nsl) issue(p, p);
  for (int s = 0; s < nsl; ++s) {
    // this wave's loads of slab s have landed once only those of the slabs after
    // it are outstanding; the barrier makes it every wave's
    asm volatile("" ::: "memory");
    if constexpr (NST == 3) {
      if (s + 1 < nsl) wait_loads<C::LPW>(); else wait_loads<0>();
    } else {
      wait_loads<0>();
    }
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (s + NST - 1 < nsl) issue(s + NST - 1, (s + NST - 1) % NST);
    const char* Ps = smem + (s % NST) * C::SLAB;
    const char* Qs = Ps + RB * KB * BLOCK;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      f16x8 ph[FT], pl[FT], qh[FT], ql[FT];
#pragma unroll
      for (int i = 0; i < FT; ++i) {
        const char* pp = Ps + ((wm * FT + i) * KB + kb) * BLOCK + lane * 16;
        const char* qp = Qs + ((wn * FT + i) * KB + kb) * BLOCK + lane * 16;
        ph[i] = *(const f16x8*)pp;
        pl[i] = *(const f16x8*)(pp + BLOCK / 2);
        qh[i] = *(const f16x8*)qp;
        ql[i] = *(const f16x8*)(qp + BLOCK / 2);
      }
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
  }
  asm volatile("" ::: "memory");
  __syncthreads();  // every wave done with the slabs before the result is staged over them

  constexpr float unscale = KIND == NS_GRAM ? 1.f / (SX * SX) : KIND == NS_POLY ? 1.f / (SA * SA) : 1.f / (SB * SX);
  float* Cs = (float*)smem;
  const int l16 = lane & 15, g4 = lane >> 4;
#pragma unroll
  for (int i = 0; i < FT; ++i)
#pragma unroll
    for (int k = 0; k < FT; ++k)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        Cs[(wm * (T / 2) + i * 16 + g4 * 4 + r) * C::CS + wn * (T / 2) + k * 16 + l16] = acc[i][k][r] * unscale;
  __syncthreads();
  // along the rows: lane l takes row l % 16, columns 8 (l / 16) .. of a 16 x 32 block
  constexpr int NB = RB * (T / 32);
  for (int b = wave; b < NB; b += 4) {
    const int rb = b / (T / 32), kb = b % (T / 32);
    float* c = Cs + (rb * 16 + l16) * C::CS + kb * 32 + g4 * 8;
    float v[8];
    *(f32x4*)v = *(const f32x4*)c;
    *(f32x4*)(v + 4) = *(const f32x4*)(c + 4);
    if constexpr (KIND == NS_GRAM) {
      store_split(M.opA + block_at(ti * RB + rb, tj * (T / 32) + kb, M.mp / 32) + lane * 16, v, SA);
    } else if constexpr (KIND == NS_POLY) {
      const int64_t at = block_at(ti * RB + rb, tj * (T / 32) + kb, M.mp / 32) + lane * 16;
      float x[8];
      load_split(M.opA + at, x, 1.f / SA);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = a.b * x[e] + a.c * v[e];
      store_split(M.opB + at, v, SB);
    } else {
      float* X = M.X + (int64_t)(ti * T + rb * 16 + l16) * M.np + tj * T + kb * 32 + g4 * 8;
      const f32x4 x0 = *(const f32x4*)X, x1 = *(const f32x4*)(X + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = a.a * x0[e] + v[e];
        v[4 + e] = a.a * x1[e] + v[4 + e];
      }
      if constexpr (KIND == NS_APPLY) {
        *(f32x4*)X = *(const f32x4*)v;
        *(f32x4*)(X + 4) = *(const f32x4*)(v + 4);
        store_split(M.opX + block_at(ti * RB + rb, tj * (T / 32) + kb, M.np / 32) + lane * 16, v, SX);
      }
    }
    if constexpr (KIND != NS_GRAM) {
      *(f32x4*)c = *(const f32x4*)v;
      *(f32x4*)(c + 4) = *(const f32x4*)(v + 4);
    }
  }
  if constexpr (SYM)
    if (ti == tj) return;  // a diagonal tile is its own mirror
  __syncthreads();
  if constexpr (KIND == NS_ORTHO || KIND == NS_MUON) {
    // to the caller's matrix, lanes along its rows
    const int64_t ld = M.tall ? M.m : M.n;
    for (int q = threadIdx.x; q < T * T; q += 256) {
      const int il = M.tall ? q % T : q / T, jl = M.tall ? q / T : q % T;
      const int i = ti * T + il, k = tj * T + jl;
      if (i >= M.m || k >= M.n) continue;
      const int64_t r = M.tall ? k : i, c = M.tall ? i : k;
      const float o = Cs[il * C::CS + jl];
      if constexpr (KIND == NS_ORTHO) {
        ((TO*)M.o)[r * M.o_stride + c] = Elem<TO>::from_f32(o);
      } else {
        const int64_t at = r * ld + c;
        const float w = M.w[at], wn = w - (M.scale * o + M.decay * w);
        M.w[at] = wn;
        if (M.o) ((TO*)M.o)[at] = Elem<TO>::from_f32(wn);
      }
    }
    return;
  }
  // along the columns: the mirrored part of a symmetric result, or X's other operand
  char* op = KIND == NS_GRAM ? M.opA : KIND == NS_POLY ? M.opB : M.opXt[a.parity ^ 1];
  constexpr float scale = KIND == NS_GRAM ? SA : KIND == NS_POLY ? SB : SX;
  for (int b = wave; b < NB; b += 4) {
    const int rb = b / (T / 32), kb = b % (T / 32);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = Cs[(kb * 32 + g4 * 8 + e) * C::CS + rb * 16 + l16];
    store_split(op + block_at(tj * RB + rb, ti * (T / 32) + kb, M.mp / 32) + lane * 16, v, scale);
  }
}

template <int T, int KB, int NST, int KIND, typename TO>
hipError_t run_product(NsArgs& a, hipStream_t st) {
  using C = NsTile<T, KB, NST>;
  static_assert(C::LDS <= 160 * 1024, "LDS of a compute unit");
  int tiles = 0;
  for (int j = 0; j < a.n; ++j) {
    a.beg[j] = tiles;
    const int tm = a.mat[j].mp / T;
    tiles += KIND == NS_GRAM || KIND == NS_POLY ? tm * (tm + 1) / 2 : tm * (a.mat[j].np / T);
  }
  a.beg[a.n] = tiles;
  const auto kern = k_ns_product<T, KB, NST, KIND, TO>;
  if (C::LDS > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kern, dim3((tiles + 7) / 8 * 8), dim3(256), C::LDS, st, a);
  return hipGetLastError();
}

template <int T, int KB, int NST>
hipError_t run_steps(NsArgs& a, bool bf16, bool muon, int steps, const float* coef, hipStream_t st) {
  for (int s = 0; s < steps; ++s) {
    a.a = coef[3 * s];
    a.b = coef[3 * s + 1];
    a.c = coef[3 * s + 2];
    a.parity = s & 1;
    hipError_t e = run_product<T, KB, NST, NS_GRAM, float>(a, st);
    if (e == hipSuccess) e = run_product<T, KB, NST, NS_POLY, float>(a, st);
    if (e != hipSuccess) return e;
    if (s + 1 < steps)
      e = run_product<T, KB, NST, NS_APPLY, float>(a, st);
    else if (muon)
      e = bf16 ? run_product<T, KB, NST, NS_MUON, __bf16>(a, st) : run_product<T, KB, NST, NS_MUON, float>(a, st);
    else
      e = bf16 ? run_product<T, KB, NST, NS_ORTHO, __bf16>(a, st) : run_product<T, KB, NST, NS_ORTHO, float>(a, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T, bool MUON>
hipError_t run_begin(NsArgs& a, hipStream_t st) {
  int blocks = 0;
  for (int j = 0; j < a.n; ++j) {
    a.beg[j] = blocks;
    a.mat[j].nssq = ns_ssq_blocks(a.mat[j].m, a.mat[j].n);
    blocks += a.mat[j].nssq;
  }
  a.beg[a.n] = blocks;
  hipLaunchKernelGGL((k_ns_begin<T, MUON>), dim3(blocks), dim3(256), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  blocks = 0;
  for (int j = 0; j < a.n; ++j) {
    a.beg[j] = blocks;
    blocks += (a.mat[j].mp / 32 * (a.mat[j].np / 32) + 3) / 4;
  }
  a.beg[a.n] = blocks;
  hipLaunchKernelGGL((k_ns_convert<T, MUON>), dim3(blocks), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

int ns_ssq_blocks(int64_t m, int64_t n) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(NS_SSQ, m * n / 2048));
}

// The edge of the result tiles for a group of matrices: the largest of 128, 64 and
// 32 whose products X X^T fill the compute units.
int ns_tile(int n, const int64_t* m) {
  for (int T : {128, 64}) {
    int64_t tiles = 0;
    for (int j = 0; j < n; ++j) {
      const int64_t tm = (m[j] + T - 1) / T;
      tiles += tm * (tm + 1) / 2;
    }
    if (tiles >= 256) return T;
  }
  return 32;
}

hipError_t launch_newton_schulz(NsArgs& a, int tile, bool bf16, bool muon, int steps, const float* coef, hipStream_t st) {
  hipError_t e = muon ? run_begin<float, true>(a, st)
                 : bf16 ? run_begin<__bf16, false>(a, st) : run_begin<float, false>(a, st);
  if (e != hipSuccess) return e;
  switch (tile) {
    case 128: return run_steps<128, 1, 2>(a, bf16, muon, steps, coef, st);
    case 64: return run_steps<64, 1, 3>(a, bf16, muon, steps, coef, st);
    default: return run_steps<32, 1, 3>(a, bf16, muon, steps, coef, st);
  }
}

}  // namespace sscn
