// Products of rows held in 8 bits (rows8.h).
//
//   forward         y = x w + bias     x [rows][k], w [k][n]: a scale for each row and 128 k,
//   input gradient  dx = dy w^T        and for each 128 x 128 of w
//   weight gradient dw = x^T dy, dbias = sum over rows of dy
//
// The first two are one product, of rows with a matrix that lies along the sum either
// way.  A result in bf16 is computed by the scaled matrix instructions, 32 x 32 x 64 on
// the codes themselves, each row's (and the matrix block's) power of two as an operand.
// Their sums are float32, but of every eight products they drop what lies below 2^-13 of
// the largest (7 2^-13 of the sum of the magnitudes at most): results are off by 1.5e-5 to
// 4e-5 of their size on sums of either sign, 3e-6 where all are positive, whatever k is: a
// hundredth of the rounding to bf16.  A result in float32 is computed by the bf16
// instructions instead, in which a code times its scale is exact and so is each product:
// 1e-7, at half the rate.
//
// The weight gradient sums over rows, whose scales differ from term to term: both operands
// become bf16 (exactly) on their way to LDS and are read from there transposed.

#include "common.h"
#include "kernels.h"
#include "rows8.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace sscn {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef int16_t i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr uint32_t NO_SOURCE = 0x80000000u;  // past every buffer: reads zero

__device__ inline u32x4 buffer_of(const void* base, uint32_t bytes) {
  const uint64_t b = (uint64_t)base;
  return u32x4{(uint32_t)b, (uint32_t)(b >> 32) & 0xffffu, bytes, 0x00020000u};
}

__device__ inline uint32_t lds_offset(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// One load per lane straight into LDS, none where s >= end: lane l's 16 bytes (4) land at
// to + 16 l (4 l), zeros where the offset lies past its buffer.  The compiler does not see the
// loads; wait_loads and the fences around the barriers order them.  The condition is in the
// block, since a branch of the compiler's would let it move the products of a loop's first
// half behind it.
template <int BYTES>
__device__ inline void load_lds(int s, int end, uint32_t to, u32x4 rsrc, uint32_t off) {
  static_assert(BYTES == 16 || BYTES == 4, "a vector or a word");
  if constexpr (BYTES == 16)
    asm volatile(
        "s_cmp_lt_i32 %0, %1\n\t"
        "s_cbranch_scc0 .Lnone%=\n\t"
        "s_mov_b32 m0, %2\n\t"
        "s_nop 0\n\t"
        "buffer_load_dwordx4 %3, %4, 0 offen lds\n\t"
        ".Lnone%=:" ::"s"(s), "s"(end), "s"(to), "v"(off), "s"(rsrc)
        : "m0", "scc");
  else
    asm volatile(
        "s_cmp_lt_i32 %0, %1\n\t"
        "s_cbranch_scc0 .Lnone%=\n\t"
        "s_mov_b32 m0, %2\n\t"
        "s_nop 0\n\t"
        "buffer_load_dword %3, %4, 0 offen lds\n\t"
        ".Lnone%=:" ::"s"(s), "s"(end), "s"(to), "v"(off), "s"(rsrc)
        : "m0", "scc");
}
// Waits for them, and for this wave's own reads of LDS.
__device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }

// Row r of the 64 that a wave's four blocks of the matrix operand cover: block j holds rows
// 16 q + 4 j + e (q, e = 0 .. 3), so that a result lane's four blocks of four values are
// sixteen neighbours of one row.
__device__ inline int interleaved(int r16, int j) { return (r16 >> 2) * 16 + j * 4 + (r16 & 3); }

// Where 16-byte chunk c of row r lies in a slab of 128-byte rows: the sixteen rows that an
// operand's read touches (consecutive ones, or interleaved ones) cover all banks once.
__device__ inline int slot_x(int r, int c) { return c ^ ((r >> 1) & 7); }
__device__ inline int slot_w(int r, int c) { return c ^ (((r >> 3) & 6) | ((r >> 1) & 1)); }

// Tile t of the result in an order in which the tiles that one XCD works on at a time (it
// gets every eighth workgroup) lie together: eight rows of tiles by as many columns.
struct TilePlace {
  int64_t m;
  int n;
};
__device__ inline TilePlace place_of(int64_t t, int64_t tiles, int64_t mt, int nt) {
  const int64_t each = (tiles + 7) / 8;
  t = (t & 7) * each + (t >> 3);
  const int64_t group = t / (8 * nt), left = t - group * 8 * nt;
  const int rows = (int)min((int64_t)8, mt - group * 8);
  return TilePlace{group * 8 + left % rows, (int)(left / rows)};
}

// Sixteen neighbouring values of a result row, from column c on.
template <typename T>
__device__ inline void store_run16(T* row, int c, int n, const float (&v)[16]) {
  T out[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) out[e] = Elem<T>::from_f32(v[e]);
  if (c + 16 <= n) {
    __builtin_memcpy(row + c, out, sizeof(out));
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (c + e < n) row[c + e] = out[e];
  }
}

// Eight neighbouring bf16 values of a result row, from column c on.
__device__ inline void store_run8(__bf16* row, int c, int n, u32x4 v, bool stream) {
  if (c + 8 <= n) {
    store_vector(row + c, v, stream);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < n) ((uint16_t*)row)[c + e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
  }
}

__device__ inline void load_bias(const float* bias, int c, int n, float (&b)[16]) {
  if (bias && c + 16 <= n) {
    __builtin_memcpy(b, bias + c, sizeof(b));
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) b[e] = bias && c + e < n ? bias[c + e] : 0.f;
  }
}

// The matrix operand's rows (result columns) that lane r of 32 reads for block j of a wave's
// 64: its result registers, rows 8 (i / 4) + 4 (lane / 32) + i % 4 of the block, are then
// sixteen neighbouring columns of one result row.
__device__ inline int interleaved32(int r, int j) { return j * 32 + ((r >> 2) & 1) * 16 + (r >> 3) * 4 + (r & 3); }
// ... and where its chunks lie (as slot_x, for those rows)
__device__ inline int slot_w32(int r, int c) { return c ^ (((r >> 1) & 3) | ((r >> 2) & 4)); }

// WX x WN waves, each TX blocks of 32 rows by 64 columns.
template <int WX_, int WN_, int TX_>
struct P8Tile {
  static constexpr int WX = WX_, WN = WN_, TX = TX_;
  static constexpr int NW = WX * WN, BM = WX * TX * 32, BN = WN * 64;
  static constexpr int SLAB = (BM + BN) * 128;
  static constexpr int XL = BM / 8 / NW, WL = BN / 8 / NW;  // loads of a wave and slab
  static constexpr int SCALES = NW * 256;                    // of four slabs: the rows', then the column blocks'
  static constexpr int LDS = 2 * SLAB + 2 * SCALES;
  // the first of a wave's nine loads that slot k of a slab's 2 TX issues
  static constexpr int at(int k) { return TX == 4 ? (k < 5 ? 2 * k : 9) : k == 0 ? 0 : k == 1 ? 3 : k == 2 ? 5 : k == 3 ? 7 : 9; }
  static_assert(XL == 4 && WL == 4 && BM / 64 < NW, "nine loads a wave and slab");
  static_assert(TX % 2 == 0 && NW * 8192 <= SLAB, "results pass through the second stage, 64 x 64 of a wave at a time");
};

// bf16 results: slabs of 128 codes through two LDS stages, multiplied in halves of 64.  A
// half's operands are read while the half before it is multiplied; a slab is loaded while
// the one before it is, and one barrier a slab says that it has arrived and that the stage
// of the one before is free.  Workgroups go on to further tiles, whose first slab is
// loaded while the results of the last one are stored.  Bound by the matrix cores' feed: 32768 x
// 4096 x 4096 450 to 535 us by the clock (2.1 to 2.4 PFLOP/s); 8192^3 403, 2.7 (the instructions
// alone, on registers, 3.9).
template <class C>
__global__ void __launch_bounds__(C::NW * 64, 2) k_product8(Product8Args a, int64_t tiles, int64_t mt, int nt) {
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wx = wave / C::WN, wn = wave % C::WN, r32 = lane & 31, h = lane >> 5;
  const uint32_t lds0 = lds_offset(smem);
  const uint32_t xstride = (uint32_t)a.x_stride, wstride = (uint32_t)a.w_stride, sstride = (uint32_t)a.xs_stride;
  const int64_t places = (tiles + 7) / 8 * 8;
  // this workgroup's next tile from place t on (places without a tile are passed over)
  auto next_tile = [&](int64_t t) {
    while (t < places && (t & 7) * (places >> 3) + (t >> 3) >= tiles) t += gridDim.x;
    return t;
  };
  int64_t m0;
  int n0;
  u32x4 rx, rw, rs;
  // A lane's row and chunk in its wave's first loads of x and w; the others are eight rows
  // further each, where the chunks' swizzle flips with the row's eights (x) and sixteens (w).
  // (Rows behind the last one lie past the buffer.)
  const int r0 = wave * C::XL * 8 + (lane >> 3), q0 = wave * C::WL * 8 + (lane >> 3);
  const uint32_t xrow = (uint32_t)r0 * xstride, wrow = (uint32_t)q0 * wstride;
  const uint32_t scale_row = wave < C::BM / 64    ? (uint32_t)(wave * 64 + lane) * sstride
                             : wave == C::BM / 64 ? (uint32_t)lane * (uint32_t)a.ws_stride
                                                  : NO_SOURCE;
  const uint32_t xk = (uint32_t)slot_x(r0, lane & 7) * 16u, wk = (uint32_t)slot_w32(q0, lane & 7) * 16u;
  u32x4 rws;
  auto set_tile = [&](int64_t t) {
    const TilePlace at = place_of(t, tiles, mt, nt);
    m0 = at.m * C::BM;
    n0 = at.n * C::BN;
    const int rows = (int)min((int64_t)C::BM, a.rows - m0), cols = min(C::BN, a.n - n0);
    rx = buffer_of(a.x + m0 * a.x_stride, (uint32_t)rows * xstride);
    rw = buffer_of(a.w + n0 * a.w_stride, (uint32_t)cols * wstride);
    rs = buffer_of(a.xs + m0 * a.xs_stride, (uint32_t)rows * sstride);
    rws = buffer_of(a.ws + (int64_t)(n0 >> 7) * a.ws_stride, (uint32_t)((cols + 127) >> 7) * (uint32_t)a.ws_stride);
  };
  // Load i of a wave for slab s: four of x, four of w, and the words with the slab's scales,
  // again with each of their four slabs (rows and blocks behind the last, and waves without
  // any: past the buffer).
  auto issue_one = [&](int s, int i) {
    const int su = __builtin_amdgcn_readfirstlane(s);
    const uint32_t st = lds0 + (su & 1) * C::SLAB + wave * 4096;
    if (i < 4) {
      const uint32_t k = (xk ^ ((i & 1) * 64u)) + (uint32_t)su * 128u;
      load_lds<16>(su, a.kb, __builtin_amdgcn_readfirstlane(st + i * 1024), rx,
                   k < xstride ? xrow + (uint32_t)i * 8u * xstride + k : NO_SOURCE);
    } else if (i < 8) {
      load_lds<16>(su, a.kb, __builtin_amdgcn_readfirstlane(st + C::BM * 128 + (i - 4) * 1024), rw,
                   wrow + (uint32_t)(i - 4) * 8u * wstride + (wk ^ ((i & 2) * 32u)) + (uint32_t)su * 128u);
    } else {
      load_lds<4>(su, a.kb,
                  __builtin_amdgcn_readfirstlane(lds0 + 2 * C::SLAB + ((su >> 2) & 1) * C::SCALES + wave * 256),
                  wave < C::BM / 64 ? rs : rws, scale_row + (uint32_t)(su & ~3));
    }
  };
  auto issue = [&](int s) {
#pragma unroll
    for (int i = 0; i < 9; ++i) issue_one(s, i);
  };
  auto operand = [&](const uint8_t* row, int slot0, int slot1) {
    union {
      i32x8 v;
      u32x4 q[2];
    } o;
    o.q[0] = *(const u32x4*)(row + slot0 * 16);
    o.q[1] = *(const u32x4*)(row + slot1 * 16);
    return o.v;
  };
  i32x8 x[C::TX], w[2][2];  // (w: of the half being multiplied, and of the next)
  uint32_t xs[C::TX], wsc;
  auto read_x = [&](int s, int half, int i) {
    const int r = (wx * C::TX + i) * 32 + r32, c = half * 4 + h * 2;
    x[i] = operand(smem + (s & 1) * C::SLAB + r * 128, slot_x(r, c), slot_x(r, c + 1));
  };
  auto read_w = [&](int s, int half, int j) {
    const int r = wn * 64 + interleaved32(r32, j), c = half * 4 + h * 2;
    w[half][j] = operand(smem + (s & 1) * C::SLAB + (C::BM + r) * 128, slot_w32(r, c), slot_w32(r, c + 1));
  };
  auto read_scale = [&](int s, int i) {
    xs[i] = smem[2 * C::SLAB + ((s >> 2) & 1) * C::SCALES + ((wx * C::TX + i) * 32 + r32) * 4 + (s & 3)];
  };
  auto read_wscale = [&](int s) {
    return (uint32_t)smem[2 * C::SLAB + ((s >> 2) & 1) * C::SCALES + C::BM * 4 + (wn >> 1) * 4 + (s & 3)];
  };
  auto arrive = [&]() {
    wait_loads();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  int64_t t = next_tile(blockIdx.x);
  if (t >= places) return;
  set_tile(t);
  issue(0);
  for (;;) {
    f32x16 acc[C::TX][2];
#pragma unroll
    for (int i = 0; i < C::TX; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = f32x16{};
    if (a.bias)  // (the sums start from it)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float b[16];
        load_bias(a.bias, n0 + wn * 64 + j * 32 + h * 16, a.n, b);
#pragma unroll
        for (int i = 0; i < C::TX; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[i][j][e] = b[e];
      }
    arrive();
#pragma unroll
    for (int l = 0; l < C::at(C::TX); ++l) issue_one(1, l);
#pragma unroll
    for (int j = 0; j < 2; ++j) read_w(0, 0, j);
#pragma unroll
    for (int i = 0; i < C::TX; ++i) {
      read_scale(0, i);
      read_x(0, 0, i);
    }
    wsc = read_wscale(0);
    auto multiply = [&](int half, int i) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[half][j], x[i], acc[i][j], 0, 0, 0, (int)wsc, 0,
                                                                    (int)xs[i]);
    };
    // Loads are dealt between the products: a wave that issues nine in a row waits for them, and
    // feeds no product meanwhile (32768 x 4096 x 4096: 552 us; four slots of three and two 514).
    auto deal = [&](int slot, int s) {  // slots 0 .. TX - 1: second halves, TX ..: the first halves behind them
#pragma unroll
      for (int l = C::at(slot); l < C::at(slot + 1); ++l) issue_one(s, l);
    };
    for (int s = 0; s < a.kb; ++s) {
      // a block of x is read again as soon as it has been multiplied
#pragma unroll
      for (int i = 0; i < C::TX; ++i) {
        if (i < 2) read_w(s, 1, i);
        multiply(0, i);
        __builtin_amdgcn_sched_barrier(0);  // (or the block would be read elsewhere, early)
        read_x(s, 1, i);
        __builtin_amdgcn_sched_barrier(0);
        deal(C::TX + i, s + 1);
      }
      uint32_t next = 0;
#pragma unroll
      for (int i = 0; i < C::TX; ++i) {
        multiply(1, i);
        __builtin_amdgcn_sched_barrier(0);
        if (i == 0) {
          arrive();
          next = read_wscale(s + 1);
        }
        // (behind the last slab: what lies in LDS, not used)
        if (i < 2) read_w(s + 1, 0, i);
        read_scale(s + 1, i);
        read_x(s + 1, 0, i);
        __builtin_amdgcn_sched_barrier(0);
        deal(i, s + 2);
      }
      wsc = next;
    }
    const int64_t m1 = m0;
    const int n1 = n0;
    t = next_tile(t + gridDim.x);
    if (t < places) {  // (every wave has read the last slab: the last barrier said so)
      set_tile(t);
      issue(0);
    }
    // 64 x 64 results of a wave at a time through its part of the second stage, from where whole
    // lines are stored: eight rows of 128 bytes by an instruction (200001 x 300 x
    // 300 52 us; from the registers, in 64 pieces of 16 bytes, 64)
    uint8_t* stage = smem + C::SLAB + wave * 8192;
#pragma unroll
    for (int p = 0; p < C::TX; p += 2) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            uint32_t v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const __bf16 lo = (__bf16)acc[p + i][j][q * 8 + e * 2], hi = (__bf16)acc[p + i][j][q * 8 + e * 2 + 1];
              v[e] = (uint32_t)__builtin_bit_cast(uint16_t, lo) | (uint32_t)__builtin_bit_cast(uint16_t, hi) << 16;
            }
            const int r = i * 32 + r32;
            *(u32x4*)(stage + r * 128 + slot_x(r, j * 4 + h * 2 + q) * 16) = u32x4{v[0], v[1], v[2], v[3]};
          }
      u32x4 line[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int r = k * 8 + (lane >> 3);
        line[k] = *(const u32x4*)(stage + r * 128 + slot_x(r, lane & 7) * 16);
      }
      const int c = n1 + wn * 64 + (lane & 7) * 8;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int64_t m = m1 + (wx * C::TX + p) * 32 + k * 8 + (lane >> 3);
        if (m < a.rows && c < a.n) store_run8((__bf16*)a.y + m * a.y_stride, c, a.n, line[k], a.stream);
      }
    }
    if (t >= places) return;
  }
}

// Sixteen codes times a power of two as sixteen bf16 values: exact from 2^-130 on, where bf16's
// smallest steps, 2^-133, are those of a code's four bits.
struct Codes16 {
  u32x4 lo, hi;
};
__device__ inline Codes16 to_bf16(u32x4 codes, float scale) {
  Codes16 o;
  uint32_t w[8];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    w[2 * q] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[q], scale, false));
    w[2 * q + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[q], scale, true));
  }
  o.lo = u32x4{w[0], w[1], w[2], w[3]};
  o.hi = u32x4{w[4], w[5], w[6], w[7]};
  return o;
}

// WX x WN waves, each 16 TX rows by 64 columns, of results in float32.
template <int WX_, int WN_, int TX_>
struct P8Exact {
  static constexpr int WX = WX_, WN = WN_, TX = TX_;
  static constexpr int NT = WX * WN * 64, BM = WX * TX * 16, BN = WN * 64;
  static constexpr int STAGE = (BM + BN) * 128, LDS = 2 * STAGE;  // 64 bf16 of every row of either operand
  static_assert(BM == BN && BM * 2 == NT, "a thread stages 32 codes of either operand");
};

// float32 results: slabs of 64 codes, made bf16 on the way to LDS.  A slab is multiplied while
// the next one is staged, between its halves, and the one behind that is on its way; an
// operand is read while the one before it is multiplied.
template <class C>
__global__ void __launch_bounds__(C::NT, 2) k_product8_exact(Product8Args a, int64_t tiles, int64_t mt, int nt) {
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wx = wave / C::WN, wn = wave % C::WN, r16 = lane & 15, g = lane >> 4;
  const int lr = threadIdx.x >> 1, lc = (threadIdx.x & 1) * 32;  // this thread's row of either operand, and its codes
  // Where this lane's chunks of its first blocks lie: x's others are 16 rows on, w's four (of
  // interleaved ones), and the second half's chunks 64 bytes off.
  const uint32_t xa = (uint32_t)((wx * C::TX * 16 + r16) * 128 + slot_x(r16, g) * 16);
  const int wr = interleaved(r16, 0);
  const uint32_t wa = (uint32_t)((C::BM + wn * 64 + wr) * 128 + slot_w(wr, g) * 16);
  const int slabs = (int)((a.x_stride + 63) / 64);
  for (int64_t t = blockIdx.x; t < (tiles + 7) / 8 * 8; t += gridDim.x) {
    if ((t & 7) * ((tiles + 7) / 8) + (t >> 3) >= tiles) continue;
    const TilePlace at = place_of(t, tiles, mt, nt);
    const int64_t m0 = at.m * C::BM;
    const int n0 = at.n * C::BN;
    const int rows = (int)min((int64_t)C::BM, a.rows - m0), cols = min(C::BN, a.n - n0);
    auto of = [&](const uint8_t* base, int64_t stride, int n) {
      return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)((uint32_t)n * (uint32_t)stride), 0x00020000);
    };
    // (rows behind the last: past the buffer)
    const auto rx = of(a.x + m0 * a.x_stride, a.x_stride, rows), rsx = of(a.xs + m0 * a.xs_stride, a.xs_stride, rows);
    const auto rw = of(a.w + n0 * a.w_stride, a.w_stride, cols);
    const auto rsw = of(a.ws + (int64_t)(n0 >> 7) * a.ws_stride, a.ws_stride, (cols + 127) >> 7);
    const uint32_t xo = (uint32_t)(lr * a.x_stride) + lc, wo = (uint32_t)(lr * a.w_stride) + lc;
    const uint32_t xso = (uint32_t)(lr * a.xs_stride), wso = (uint32_t)(lr >> 7) * (uint32_t)a.ws_stride;
    struct Staged {
      u32x4 x[2], w[2];
      uint32_t sx, sw;
    };
    auto fetch = [&](Staged& o, int s) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t k = (uint32_t)s * 64u + h * 16u;
        const bool in = k + lc < (uint32_t)a.x_stride;
        o.x[h] = __builtin_amdgcn_raw_buffer_load_b128(rx, (int)(in ? xo + k : NO_SOURCE), 0, 0);
        o.w[h] = __builtin_amdgcn_raw_buffer_load_b128(rw, (int)(in ? wo + k : NO_SOURCE), 0, 0);
      }
      const uint32_t b = (uint32_t)min(s, slabs - 1) >> 1;
      o.sx = __builtin_amdgcn_raw_buffer_load_b8(rsx, (int)(xso + b), 0, 0);
      o.sw = __builtin_amdgcn_raw_buffer_load_b8(rsw, (int)(wso + b), 0, 0);
    };
    auto put = [&](const Staged& o, int st) {
      uint8_t* X = smem + st * C::STAGE + lr * 128;
      uint8_t* W = X + C::BM * 128;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = lc / 8 + h * 2;
        const Codes16 vx = to_bf16(o.x[h], row8_pow2(o.sx)), vw = to_bf16(o.w[h], row8_pow2(o.sw));
        *(u32x4*)(X + slot_x(lr, c) * 16) = vx.lo;
        *(u32x4*)(X + slot_x(lr, c + 1) * 16) = vx.hi;
        *(u32x4*)(W + slot_w(lr, c) * 16) = vw.lo;
        *(u32x4*)(W + slot_w(lr, c + 1) * 16) = vw.hi;
      }
    };
    f32x4 acc[C::TX][4];
    {  // the sums start from the bias
      float b[16];
      load_bias(a.bias, n0 + wn * 64 + g * 16, a.n, b);
#pragma unroll
      for (int i = 0; i < C::TX; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{b[4 * j], b[4 * j + 1], b[4 * j + 2], b[4 * j + 3]};
    }
    Staged ahead;
    fetch(ahead, 0);
    __syncthreads();  // (every wave is done with the tile before)
    put(ahead, 0);
    fetch(ahead, 1);
    for (int s = 0; s < slabs; ++s) {
      const int st = s & 1;
      __syncthreads();
      bf16x8 x[2], w[2][4];
      const uint8_t* base = smem + st * C::STAGE;
      auto x_read = [&](int n) {
        x[n & 1] = *(const bf16x8*)(base + (xa ^ (n / C::TX * 64u)) + n % C::TX * 2048);
      };
      auto w_read = [&](int half, int j) { w[half][j] = *(const bf16x8*)(base + (wa ^ (half * 64u)) + j * 512); };
#pragma unroll
      for (int j = 0; j < 4; ++j) w_read(0, j);
      x_read(0);
#pragma unroll
      for (int n = 0; n < 2 * C::TX; ++n) {
        const int half = n / C::TX, i = n % C::TX;
        if (n + 1 < 2 * C::TX) x_read(n + 1);
        if (half == 0 && i >= C::TX - 4) w_read(1, i - (C::TX - 4));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[half][j], x[n & 1], acc[i][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        if (n == C::TX - 1) {
          put(ahead, st ^ 1);  // (behind the last slab: zeros, not read)
          fetch(ahead, s + 2);
        }
      }
    }
    // 16 x 64 results of a wave at a time through LDS, from where whole lines are stored
    __syncthreads();
    uint8_t* stage = smem + wave * 4096;
    const int c = n0 + wn * 64 + (lane & 15) * 4;
#pragma unroll
    for (int i = 0; i < C::TX; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) *(f32x4*)(stage + r16 * 256 + ((g * 4 + j) ^ r16) * 16) = acc[i][j];
      f32x4 line[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int r = k * 4 + g;
        line[k] = *(const f32x4*)(stage + r * 256 + (r16 ^ r) * 16);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int64_t m = m0 + (wx * C::TX + i) * 16 + k * 4 + g;
        if (m >= a.rows || c >= a.n) continue;
        float* y = (float*)a.y + m * a.y_stride + c;
        if (c + 4 <= a.n) {
          store_vector(y, line[k], a.stream);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (c + e < a.n) y[e] = line[k][e];
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Few rows: a workgroup's waves share the sum of MB x 16 rows by NB x 16 columns, every wave
// a run of its blocks of 128, operands straight into registers (16 rows of 128 bytes by two
// loads), and meet in LDS.  Bound by latency and by reading the matrix once: one row, 300 ->
// 3755, 3.0 us; a call of 1 x 4096 x 4096 5.4 (in 128 x 128 tiles 19.7).
constexpr int FEW_WAVES = 8;

template <typename T, int MB, int NB>
__global__ void __launch_bounds__(FEW_WAVES * 64) k_product8_few(Product8Args a, int nt) {
  constexpr int CS = NB * 16 + 4;  // floats of a staged row
  __shared__ __attribute__((aligned(16))) float sums[FEW_WAVES][MB * 16][CS];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int r16 = lane & 15, g = lane >> 4;
  const int tn = blockIdx.x % nt;
  const int64_t m0 = (int64_t)(blockIdx.x / nt) * (MB * 16);
  const int n0 = tn * (NB * 16);
  const int b0 = a.kb * wave / FEW_WAVES, b1 = a.kb * (wave + 1) / FEW_WAVES;
  const uint8_t* x[MB];
  const uint8_t* xs[MB];
  const uint8_t* w[NB];
#pragma unroll
  for (int i = 0; i < MB; ++i) {  // (rows and columns behind the last: the last one, not stored)
    const int64_t m = min(m0 + i * 16 + r16, a.rows - 1);
    x[i] = a.x + m * a.x_stride + g * 32;
    xs[i] = a.xs + m * a.xs_stride;
  }
#pragma unroll
  for (int j = 0; j < NB; ++j) w[j] = a.w + (int64_t)min(n0 + j * 16 + r16, a.n - 1) * a.w_stride + g * 32;
  const uint8_t* ws = a.ws + (int64_t)(n0 >> 7) * a.ws_stride;
  struct Block {
    u32x4 x[MB][2], w[NB][2];
    uint32_t xs[MB], ws;
  };
  auto load = [&](Block& o, int b) {
    const int k = b * 128 + g * 32;
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) o.w[j][h] = *(const u32x4*)(w[j] + b * 128 + h * 16);
#pragma unroll
    for (int i = 0; i < MB; ++i) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        o.x[i][h] = k + h * 16 < a.x_stride ? *(const u32x4*)(x[i] + b * 128 + h * 16) : u32x4{0, 0, 0, 0};
      o.xs[i] = xs[i][b];
    }
    o.ws = ws[b];
  };
  f32x4 acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](const Block& o) {
    if constexpr (sizeof(T) == 2) {
      union {
        u32x4 h[2];
        i32x8 v;
      } p, q;
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        p.h[0] = o.w[j][0];
        p.h[1] = o.w[j][1];
#pragma unroll
        for (int i = 0; i < MB; ++i) {
          q.h[0] = o.x[i][0];
          q.h[1] = o.x[i][1];
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(p.v, q.v, acc[i][j], 0, 0, 0, (int)o.ws, 0,
                                                                       (int)o.xs[i]);
        }
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        Codes16 cw[NB], cx[MB];
#pragma unroll
        for (int j = 0; j < NB; ++j) cw[j] = to_bf16(o.w[j][h], row8_pow2(o.ws));
#pragma unroll
        for (int i = 0; i < MB; ++i) cx[i] = to_bf16(o.x[i][h], row8_pow2(o.xs[i]));
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int i = 0; i < MB; ++i) {
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, cw[j].lo),
                                                                __builtin_bit_cast(bf16x8, cx[i].lo), acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, cw[j].hi),
                                                                __builtin_bit_cast(bf16x8, cx[i].hi), acc[i][j], 0, 0, 0);
          }
      }
    }
  };
  constexpr int DEPTH = MB + NB <= 2 ? 4 : 2;  // blocks in flight
  int b = b0;
  for (; b + DEPTH <= b1; b += DEPTH) {
    Block o[DEPTH];
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) load(o[d], b + d);
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) multiply(o[d]);
  }
  for (; b < b1; ++b) {
    Block o;
    load(o, b);
    multiply(o);
  }
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) *(f32x4*)&sums[wave][i * 16 + r16][j * 16 + g * 4] = acc[i][j];
  __syncthreads();
  for (int v = threadIdx.x; v < MB * 16 * NB * 16; v += FEW_WAVES * 64) {
    const int r = v / (NB * 16), c = v % (NB * 16);
    if (m0 + r >= a.rows || n0 + c >= a.n) continue;
    float s = a.bias ? a.bias[n0 + c] : 0.f;
#pragma unroll
    for (int k = 0; k < FEW_WAVES; ++k) s += sums[k][r][c];
    ((T*)a.y)[(m0 + r) * a.y_stride + n0 + c] = Elem<T>::from_f32(s);
  }
}

// ---------------------------------------------------------------------------
// weight gradient

constexpr int WG_ROWS = 64;        // rows of a slab
constexpr int PANEL = WG_ROWS * 256;  // bytes of its 128 columns in bf16

// Eight rows' values of one column of a staged panel [64 rows][128 bf16], for each lane: the
// lanes of a 16-lane group read rows 8 g .. + 3 (then + 4 .. 7) in pieces of four columns,
// 16 apart, and get them transposed: lane 4 q + e column 16 (unit + q) + 4 j + e.  A piece of
// 8 bytes lies where the 32 lanes that read together, and the 16 that write 16 bytes each,
// cover all banks once.
__device__ inline int piece_at(int row, int unit, int sub) {
  return row * 256 + (unit ^ ((row >> 1) & 4) ^ (row & 1)) * 32 + (sub ^ (row & 3)) * 8;
}
// at: piece_at of the lane's row and column piece; four rows on, the swizzle is the same.
__device__ inline bf16x8 column_operand(uint32_t at) {
  typedef __attribute__((address_space(3))) i16x4* P;
  union {
    i16x4 h[2];
    bf16x8 v;
  } o;
  o.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)at);
  o.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)(at + 4 * 256));
  return o.v;
}
// WK x WN waves, each 16 TK rows of dw by 64 columns.
template <int WK_, int WN_, int TK_>
struct Wg8Tile {
  static constexpr int WK = WK_, WN = WN_, TK = TK_;
  static constexpr int NT = WK * WN * 64, BK = WK * TK * 16, BN = WN * 64;
  static constexpr int STAGE = (BK + BN) / 128 * PANEL, LDS = 2 * STAGE;
  static_assert(BK == BN && BK * 2 == NT, "a thread stages 32 codes of either operand");
};

// A tile of dw over a run of rows: slabs of 64 rows through two LDS stages.  Bound by reading the
// transposed operands, which takes LDS about as long as the products take the matrix cores:
// 32768 x 4096 x 4096 926 to 970 us, 1.13 to 1.19 PFLOP/s.
template <class C>
__global__ void __launch_bounds__(C::NT, 2) k_weight_grad8(WeightGrad8Args a, int kt, int nt, int splits) {
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wk = wave / C::WN, wn = wave % C::WN, r16 = lane & 15, g = lane >> 4;
  const int split = blockIdx.x / (kt * nt), tile = blockIdx.x - split * (kt * nt);
  const int tk = tile / nt, tn = tile - tk * nt;
  const int64_t slabs = (a.rows + WG_ROWS - 1) / WG_ROWS;
  const int64_t s0 = slabs * split / splits, s1 = slabs * (split + 1) / splits;
  // Staging: this thread's 32 codes of a row of either operand (zeros behind the last row and
  // column: past the buffer, whose end is the last row's within a slab).
  const int panel = threadIdx.x >> 8, lr = (threadIdx.x & 255) >> 2, lc = (threadIdx.x & 3) * 32;
  const int xc = tk * C::BK + panel * 128 + lc, yc = tn * C::BN + panel * 128 + lc;
  uint32_t xo[2], yo[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    xo[h] = xc + h * 16 < a.x_stride ? (uint32_t)(lr * a.x_stride + xc + h * 16) : NO_SOURCE;
    yo[h] = yc + h * 16 < a.dy_stride ? (uint32_t)(lr * a.dy_stride + yc + h * 16) : NO_SOURCE;
  }
  // (scales of blocks behind the last: the last one's, for codes that are zero)
  const uint32_t xso = (uint32_t)(lr * a.xs_stride + (min(xc, a.k - 1) >> 7));
  const uint32_t yso = (uint32_t)(lr * a.dys_stride + (min(yc, a.n - 1) >> 7));
  struct Staged {
    u32x4 x[2], y[2];
    uint32_t sx, sy;
  };
  auto fetch = [&](Staged& o, int64_t s) {
    const int rows = (int)(s < s1 ? min((int64_t)WG_ROWS, a.rows - s * WG_ROWS) : 0);
    const int64_t m = (s < s1 ? s : s0) * WG_ROWS;
    auto of = [&](const uint8_t* base, int64_t stride) {
      return __builtin_amdgcn_make_buffer_rsrc((void*)(base + m * stride), 0, (int)((uint32_t)rows * (uint32_t)stride),
                                               0x00020000);
    };
    const auto rx = of(a.x, a.x_stride), ry = of(a.dy, a.dy_stride), rsx = of(a.xs, a.xs_stride), rsy = of(a.dys, a.dys_stride);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      o.x[h] = __builtin_amdgcn_raw_buffer_load_b128(rx, (int)xo[h], 0, 0);
      o.y[h] = __builtin_amdgcn_raw_buffer_load_b128(ry, (int)yo[h], 0, 0);
    }
    o.sx = __builtin_amdgcn_raw_buffer_load_b8(rsx, (int)xso, 0, 0);
    o.sy = __builtin_amdgcn_raw_buffer_load_b8(rsy, (int)yso, 0, 0);
  };
  // Sixteen codes at a time (a unit), two pieces to a store: an odd row's swizzle exchanges
  // the pieces of each pair, an exchange of words while they are codes.
  const uint32_t lds0 = lds_offset(smem), at0 = (uint32_t)(panel * PANEL + piece_at(lr, lc / 16, 0) - (lr & 1) * 8);
  auto put = [&](const Staged& o, int st) {
    uint8_t* to = smem + st * C::STAGE;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int of_y = 0; of_y < 2; ++of_y) {
        const u32x4 c = of_y ? o.y[h] : o.x[h];
        const u32x4 d = lr & 1 ? u32x4{c[1], c[0], c[3], c[2]} : c;
        const Codes16 v = to_bf16(d, row8_pow2(of_y ? o.sy : o.sx));
        // (unit and pair of pieces: bits 5 and 4 of the place)
        *(u32x4*)(to + of_y * (C::BK / 128 * PANEL) + (at0 ^ (h * 32))) = v.lo;
        *(u32x4*)(to + of_y * (C::BK / 128 * PANEL) + (at0 ^ (h * 32 + 16))) = v.hi;
      }
  };
  f32x4 acc[C::TK][4], bacc[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    bacc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < C::TK; ++i) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const bool bias = a.db && tk == 0 && wk == 0;
  bf16x8 one;
#pragma unroll
  for (int e = 0; e < 8; ++e) one[e] = (__bf16)1.f;
  // Where this lane's pieces of its wave's columns lie, 64 of them at a time (half a panel;
  // the other half is 128 bytes off), in each of the four interleaved blocks.
  const int row0 = g * 8 + (r16 >> 2), xh = C::TK == 8 ? 0 : wk & 1;
  uint32_t xa[4], ya[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    xa[j] = lds0 + (wk * C::TK / 8) * PANEL + piece_at(row0, xh * 4 + (r16 & 3), j);
    ya[j] = lds0 + C::BK / 128 * PANEL + (wn >> 1) * PANEL + piece_at(row0, (wn & 1) * 4 + (r16 & 3), j);
  }
  // Slab s is multiplied while the next one is staged, between its halves, and the one
  // behind that is on its way: a trip through memory has a whole slab's time.
  Staged ahead;
  if (s0 < s1) {
    fetch(ahead, s0);
    put(ahead, 0);
    fetch(ahead, s0 + 1);
  }
  // with_bias: the waves that also sum dy (a loop of their own: a branch in it would let the
  // products move behind it)
  auto loop = [&](auto with_bias) {
    for (int64_t s = s0; s < s1; ++s) {
      const int st = (int)(s - s0) & 1;
      __syncthreads();
      bf16x8 x[2], y[2][4];
      auto x_read = [&](int n) {  // block n % TK of 32 rows n / TK
        const int i = n % C::TK;
        x[n & 1] = column_operand((xa[i & 3] ^ ((i >> 2) * 128)) + st * C::STAGE + n / C::TK * 32 * 256);
      };
      auto y_read = [&](int mb, int j) { y[mb][j] = column_operand(ya[j] + st * C::STAGE + mb * 32 * 256); };
#pragma unroll
      for (int j = 0; j < 4; ++j) y_read(0, j);
      x_read(0);
#pragma unroll
      for (int n = 0; n < 2 * C::TK; ++n) {
        const int mb = n / C::TK, i = n % C::TK;
        // an operand is read while the one before it is multiplied
        if (n + 1 < 2 * C::TK) x_read(n + 1);
        if (mb == 0 && i >= C::TK - 4) y_read(1, i - (C::TK - 4));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y[mb][j], x[n & 1], acc[i][j], 0, 0, 0);
        if (decltype(with_bias)::value && i == C::TK - 1)
#pragma unroll
          for (int j = 0; j < 4; ++j) bacc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y[mb][j], one, bacc[j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        if (n == C::TK - 1) {
          put(ahead, st ^ 1);  // (behind the last slab: zeros, not read)
          fetch(ahead, s + 2);
        }
      }
    }
  };
  if (bias)
    loop(std::true_type{});
  else
    loop(std::false_type{});
  // lane: rows k of the wave's as the pieces interleave them, columns n = 16 g .. + 15
  float* out = a.part ? a.part + (int64_t)split * a.k * a.n : a.dw;
  const int64_t stride = a.part ? a.n : a.dw_stride;
  const int c = tn * C::BN + wn * 64 + g * 16;
#pragma unroll
  for (int i = 0; i < C::TK; ++i) {
    const int k = tk * C::BK + wk * (C::TK * 16) + (i >> 2) * 64 + interleaved(r16, i & 3);
    if (k >= a.k || c >= a.n) continue;
    float v[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = acc[i][e >> 2][e & 3];
    store_run16<float>(out + (int64_t)k * stride, c, a.n, v);
  }
  if (bias && r16 == 0 && c < a.n) {
    float v[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = bacc[e >> 2][e & 3];
    store_run16<float>(a.part ? a.part + (int64_t)splits * a.k * a.n + (int64_t)split * a.n : a.db, c, a.n, v);
  }
}

// The partial tiles added in order; row k of the grid is the bias gradient.
__global__ void __launch_bounds__(256) k_weight_grad8_sum(WeightGrad8Args a, int splits) {
  const int64_t size = (int64_t)a.k * a.n;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < size + (a.db ? a.n : 0); i += (int64_t)gridDim.x * 256) {
    const bool bias = i >= size;
    const float* p = bias ? a.part + splits * size + (i - size) : a.part + i;
    const int64_t step = bias ? a.n : size;
    float v = 0.f;
#pragma unroll 8
    for (int s = 0; s < splits; ++s) v += p[s * step];
    if (bias)
      a.db[i - size] = v;
    else
      a.dw[i / a.n * a.dw_stride + i % a.n] = v;
  }
}

template <class C>
hipError_t launch_tiles(const Product8Args& a, int workgroups, hipStream_t st) {
  const int64_t mt = (a.rows + C::BM - 1) / C::BM;
  const int nt = (a.n + C::BN - 1) / C::BN;
  const int64_t tiles = mt * nt;
  const hipError_t e = allow_lds<k_product8<C>>(C::LDS);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_product8<C>, dim3((unsigned)std::min<int64_t>((tiles + 7) / 8 * 8, workgroups)), dim3(C::NW * 64),
                     C::LDS, st, a, tiles, mt, nt);
  return hipGetLastError();
}

}  // namespace

template <typename T>
hipError_t launch_few(const Product8Args& a, hipStream_t st) {
  auto go = [&](auto kernel, int mb, int nb) {
    const int nt = (a.n + nb * 16 - 1) / (nb * 16);
    hipLaunchKernelGGL(kernel, dim3((unsigned)((a.rows + mb * 16 - 1) / (mb * 16) * nt)), dim3(FEW_WAVES * 64), 0, st, a, nt);
    return hipGetLastError();
  };
  if (a.rows <= 16) return go(k_product8_few<T, 1, 1>, 1, 1);
  if (a.rows <= 32) return go(k_product8_few<T, 2, 1>, 2, 1);
  if (a.rows <= 64) return go(k_product8_few<T, 2, 2>, 2, 2);  // (64 x 4096 x 4096: 12.0 us, 64 x 32 17.7)
  return go(k_product8_few<T, 4, 2>, 4, 2);
}

template <class C>
hipError_t launch_exact(const Product8Args& a, hipStream_t st) {
  const int64_t mt = (a.rows + C::BM - 1) / C::BM;
  const int nt = (a.n + C::BN - 1) / C::BN;
  const int64_t tiles = mt * nt;
  const hipError_t e = allow_lds<k_product8_exact<C>>(C::LDS);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_product8_exact<C>, dim3((unsigned)std::min<int64_t>((tiles + 7) / 8 * 8, 1 << 20)), dim3(C::NT),
                     C::LDS, st, a, tiles, mt, nt);
  return hipGetLastError();
}

hipError_t launch_product8(bool bf16, const Product8Args& a, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  // Few rows, or results of few tiles (by 64 x 32), go to the kernel whose waves share a sum:
  // 1 x 4096 x 4096 5.4 us, in 128 x 128 tiles 19.7; 128 x 4096 x 4096 (256 tiles) 17.7 and 22,
  // in float32 18.7 and 54; 256 x 4096 x 4096 (512) 33.6 and 22, in float32 35 and 55.
  const int64_t few = (a.rows + 63) / 64 * ((a.n + 31) / 32);
  if (a.rows <= 32 || few <= (bf16 ? 256 : 512)) return bf16 ? launch_few<__bf16>(a, st) : launch_few<float>(a, st);
  // Rounds of workgroups times what one takes, in us for `slabs` slabs, as measured: 256 x 256
  // tiles, one a compute unit, and 128 x 128, two.  32768 x 4096 x 4096 bf16 502 and 675 us,
  // float32 950 and 1152; 32768 x 512 x 4096 bf16 143 and 114; 200001 x 300 x 300 bf16 82 and
  // 52, float32 129 and 120; 2000 x 2000 x 2000 bf16 26 and 16, float32 59 and 30.
  const double big = (double)(((a.rows + 255) / 256 * ((a.n + 255) / 256) + 255) / 256);
  const double small = (double)(((a.rows + 127) / 128 * ((a.n + 127) / 128) + 511) / 512);
  if (bf16) {
    if (big * (11.0 + 1.68 * a.kb) < small * (2.1 + 1.25 * a.kb)) return launch_tiles<P8Tile<2, 4, 4>>(a, 256, st);
    return launch_tiles<P8Tile<2, 2, 2>>(a, 512, st);
  }
  const double slabs = (double)((a.x_stride + 63) / 64);
  if (big * (9.0 + 1.73 * slabs) < small * (5.0 + 1.07 * slabs)) return launch_exact<P8Exact<2, 4, 8>>(a, st);
  return launch_exact<P8Exact<2, 2, 4>>(a, st);
}

namespace {

typedef Wg8Tile<2, 4, 8> WgBig;
typedef Wg8Tile<2, 2, 4> WgSmall;

int64_t tiles_of(int64_t k, int64_t n, int side) { return (k + side - 1) / side * ((n + side - 1) / side); }

// Workgroups that share a tile's rows, at most: as many as the compute units hold at once (one of
// 256 x 256 or two of 128 x 128 each), with two slabs of rows at least.
int most_splits(int64_t rows, int64_t k, int64_t n, bool big) {
  const int64_t slabs = (rows + WG_ROWS - 1) / WG_ROWS, held = big ? 256 : 512;
  return (int)std::max<int64_t>(1, std::min<int64_t>(slabs / 2, held / tiles_of(k, n, big ? 256 : 128)));
}

// The tile, and how many workgroups share the rows: the plan whose rounds of workgroups and
// partial results, written and read at 5 TB/s, take least, in us fitted to measured times (a slab
// of 64 rows 1.8 in 256 x 256 tiles, 1.4 in 128 x 128).  32768 x 4096 x 4096: 950 in 256 x 256
// tiles, 1385 in 128 x 128; 20000 x 300 x 300: 44 and 28; 1 x 300 x 3755: 15 and 8.
struct WgPlan {
  bool big;
  int splits;
};
WgPlan plan_weight_grad8(int64_t rows, int64_t k, int64_t n) {
  const double slabs = (double)((rows + WG_ROWS - 1) / WG_ROWS), part = (double)k * (double)n * 8.0 / 5e6;
  WgPlan best{false, 1};
  double least = 1e300;
  for (int big = 0; big < 2; ++big) {
    const int64_t tiles = tiles_of(k, n, big ? 256 : 128), held = big ? 256 : 512;
    const double slab = big ? 1.8 : 1.4;
    // slab * slabs / s + part * s is least at this s; divided rows take one round
    const int s = (int)std::lround(
        std::min(std::max(std::sqrt(slab * slabs / part), 1.0), (double)most_splits(rows, k, n, big != 0)));
    for (int splits : {1, s}) {
      const double t = (double)((tiles * splits + held - 1) / held) * (5.0 + slab * std::ceil(slabs / splits)) +
                       (splits > 1 ? 3.0 + part * splits : 0.0);
      if (t < least) {
        least = t;
        best = WgPlan{big != 0, splits};
      }
    }
  }
  return best;
}

template <class C>
hipError_t weight_grad8(const WeightGrad8Args& a, int splits, hipStream_t st) {
  const int kt = (a.k + C::BK - 1) / C::BK, nt = (a.n + C::BN - 1) / C::BN;
  const hipError_t e = allow_lds<k_weight_grad8<C>>(C::LDS);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_weight_grad8<C>, dim3((unsigned)(kt * nt * splits)), dim3(C::NT), C::LDS, st, a, kt, nt, splits);
  return hipGetLastError();
}

}  // namespace

int32_t weight_grad8_most_splits(int64_t rows, int32_t k, int32_t n) {
  return std::max(most_splits(rows, k, n, false), most_splits(rows, k, n, true));
}

hipError_t launch_weight_grad8(const WeightGrad8Args& args, hipStream_t st) {
  WeightGrad8Args a = args;
  const WgPlan plan = plan_weight_grad8(a.rows, a.k, a.n);
  if (plan.splits == 1) a.part = nullptr;
  const hipError_t e =
      plan.big ? weight_grad8<WgBig>(a, plan.splits, st) : weight_grad8<WgSmall>(a, plan.splits, st);
  if (e != hipSuccess || plan.splits == 1) return e;
  const int64_t size = (int64_t)a.k * a.n + (a.db ? a.n : 0);
  hipLaunchKernelGGL(k_weight_grad8_sum, dim3((unsigned)std::min<int64_t>((size + 255) / 256, 4096)), dim3(256), 0, st, a,
                     plan.splits);
  return hipGetLastError();
}

}  // namespace sscn
