// Normalisation over the rows of a sample and the channels of a group, with an
// activation, forward and backward; rows are sites, channels last.
//
//   mean = sum x / n,  r = 1 / sqrt(sum (x - mean)^2 / n + eps)   over a sample and group
//   h = (x - mean) r,  z = h gain + shift,  y = act(z)
//   backward  dz = dy act'(z), t = dz gain, dx = r (t - sum t / n - h sum(t h) / n),
//             dgain = sum over rows of dz h, dshift = sum over rows of dz
//
// Memory-bound.  Samples are runs of rows of any lengths, known on the device only.
//
// Samples that are small on average: one launch, a workgroup for a sample and a slice of
// whole groups, its rows in registers (k_group_norm_small, k_group_norm_bwd_small).  A
// sample that is larger than that is read again for each step, still by that workgroup:
// 20011 rows of 100 in bf16, 100 equal samples 35 us forward and 31 backward, one of them with
// nine tenths of the rows 147 and 280; 200000 rows in 1000 samples 88 forward, and 2834.
//
// Larger ones: work is dealt by equal chunks of rows, and a workgroup walks through the
// samples that its chunk meets.  The part of sample s in chunk c is piece c + s, which
// numbers all pieces without a scan.  Three launches: sums of each piece, sums of each
// sample, the result.  The last one goes through the chunks backwards, so that it finds in
// the last-level cache what the first one read last.  Where a sample has few pieces on average, the
// last launch sums them itself, every workgroup those of the samples that it meets; a sample
// with most of the rows then costs more (200001 rows of 300 in bf16: 100 equal samples 78 us forward
// and 117 backward, one of them with nine tenths of the rows 96 and 232).
//
// A thread owns one vector of V columns and every rpb-th row.  The last vector starts V
// columns before the end, where its first `skip` columns repeat those of the vector
// before (left out of every sum and not stored).  Variances: in registers from the
// deviations themselves; in streams a thread sums deviations from its own first value of a
// column, which cannot cancel by more than the number of its rows, and threads, pieces and
// columns are joined by their means.  Every sum is taken in an order that sizes alone
// decide.  All arithmetic is float32.

#include "common.h"
#include "kernels.h"
#include "lanes.h"
#include "norm_rules.h"
#include "rows8.h"

namespace sscn {

namespace {

template <typename T, int V>
struct Pack {
  T e[V];
};
template <typename T, int V>
__device__ inline Pack<T, V> load_pack(const T* p) {
  Pack<T, V> v;
  __builtin_memcpy(&v, p, sizeof(v));
  return v;
}
// All but the first `skip` elements: those are another thread's, which may still have to
// read what lies there (a result may take its input's place).
template <typename T, int V>
__device__ inline void store_pack(T* p, const float (&f)[V], int skip, bool stream) {
  Pack<T, V> v;
#pragma unroll
  for (int e = 0; e < V; ++e) v.e[e] = Elem<T>::from_f32(f[e]);
  if (skip == 0) {
    if constexpr (sizeof(v) >= 4)
      store_vector(p, v, stream);
    else
      *p = v.e[0];
    return;
  }
  if constexpr (V >= 8)
    if (V - skip >= 4) __builtin_memcpy(p + V - 4, v.e + V - 4, 4 * sizeof(T));
#pragma unroll
  for (int e = 1; e < V; ++e)
    if (e >= skip && (V < 8 || e < V - 4 || V - skip < 4)) p[e] = v.e[e];
}

// What a thread holds of a row: V elements, or V codes and their scales.
template <typename T, int V, bool X8>
struct Held {
  Pack<T, V> v;
  __device__ inline void values(float (&f)[V], int) const {
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = Elem<T>::to_f32(v.e[e]);
  }
};
template <typename T, int V>
struct Held<T, V, true> {
  uint32_t c[(V + 3) / 4];
  uint8_t s[2];  // the scales of its two blocks
  // split: elements before the next scale's block
  __device__ inline void values(float (&f)[V], int split) const {
    const float s0 = row8_pow2(s[0]), s1 = row8_pow2(s[1]);
    if constexpr (V == 1) {
      float t[4];
      row8_values4(c[0], s0, t);
      f[0] = t[0];
    } else if (split >= V) {
#pragma unroll
      for (int q = 0; q < V; q += 4) row8_values4(c[q / 4], s0, f + q);
    } else {
#pragma unroll
      for (int q = 0; q < V; q += 4) row8_values4(c[q / 4], 1.f, f + q);
#pragma unroll
      for (int e = 0; e < V; ++e) f[e] *= e < split ? s0 : s1;
    }
  }
};

// Where a thread's rows lie: `at` its first one's vector, `step` bytes from one of its rows to
// the next.
template <typename T, int V>
struct From {
  const char* at;
  int64_t step;
  __device__ inline From(const void* base, int64_t stride, int64_t row, int col, int rpb)
      : at((const char*)base + (row * stride + col) * (int64_t)sizeof(T)), step(stride * (int64_t)sizeof(T) * rpb) {}
  __device__ inline void load(Pack<T, V>& v, int k) const { v = load_pack<T, V>((const T*)(at + k * step)); }
  __device__ inline T* put(int k) const { return (T*)(const_cast<char*>(at) + k * step); }
};
template <typename T, int V, bool X8>
struct FromX {
  From<T, V> f;
  __device__ inline FromX(const GroupNormArgs& a, int64_t row, int col, int, int rpb)
      : f(a.x, a.x_stride, row, col, rpb) {}
  __device__ inline void load(Held<T, V, X8>& h, int k) const { f.load(h.v, k); }
};
template <typename T, int V>
struct FromX<T, V, true> {
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t step, sstep;
  int split;
  __device__ inline FromX(const GroupNormArgs& a, int64_t row, int col, int split, int rpb) : split(split) {
    const int64_t cs = row8_code_stride(a.cols), ss = row8_scale_stride(a.cols);
    codes = a.codes + row * cs + col;
    scales = a.scales + row * ss + (col >> 7);
    step = cs * rpb;
    sstep = ss * rpb;
  }
  __device__ inline void load(Held<T, V, true>& h, int k) const {
    h.c[0] = 0;
    __builtin_memcpy(h.c, codes + k * step, V);
    const uint8_t* p = scales + k * sstep;
    h.s[0] = p[0];
    h.s[1] = p[split < V ? 1 : 0];
  }
};

// Every operation is rounded by itself: forward and backward take the same branch of the
// activation, and so does any program that follows the formula in float32.
__device__ inline float normal(float x, float mean, float r) {
#pragma clang fp contract(off)
  return (x - mean) * r;
}
__device__ inline float affine(float h, float gain, float shift) {
#pragma clang fp contract(off)
  const float p = h * gain;
  return p + shift;
}
__device__ inline float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }
template <bool SILU>
__device__ inline float activated(float z, float slope) {
  if constexpr (SILU) return z * sigmoid(z);
  const float below = slope == 0.f ? 0.f : slope * z;
  return z < 0.f ? below : z;
}
// dy act'(z).  The framework's rule at zero: a rectifier's derivative is 0 there, the leaky
// one's 1.
template <bool SILU>
__device__ inline float gradient(float dy, float h, float gain, float shift, float slope) {
  const float z = affine(h, gain, shift);
  if constexpr (SILU) {
    const float s = sigmoid(z);
    return dy * (s * (1.f + z * (1.f - s)));
  }
  return (slope == 0.f ? z > 0.f : z >= 0.f) ? dy : dy * slope;
}

__device__ inline int64_t sample_begin(const GroupNormArgs& a, int s) { return a.begin ? a.begin[s] : s * a.span; }

// The last sample that starts at row r or before it (-1: none; batch: r lies behind the
// last one), and its rows, by a whole wave: 256 probes a round, all in flight.  Bounds hold
// for any offsets.
struct Span {
  int s;
  int64_t begin, end;
};
__device__ inline Span span_of(const GroupNormArgs& a, int64_t r) {
  if (!a.begin) {
    const int s = (int)(r / a.span);
    return Span{s, s * a.span, (s + 1) * a.span};
  }
  const int lane = threadIdx.x & 63;
  int lo = -1, hi = a.batch + 1;
  int32_t begin = 0, end = 0;
  while (hi - lo > 1) {
    const int step = (hi - lo - 1 + 255) / 256;
    int32_t v[4];
    uint32_t at[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // (below 2^31 + 256 steps: no overflow)
      at[i] = (uint32_t)(lo + 1) + (uint32_t)(i * 64 + lane) * (uint32_t)step;
      v[i] = a.begin[min(at[i], (uint32_t)a.batch)];
    }
    int m = 0;  // probes at r or before it
#pragma unroll
    for (int i = 0; i < 4; ++i) m += __popcll(__ballot(at[i] < (uint32_t)hi && v[i] <= r));
    auto probe = [&](int k) {
      return __builtin_amdgcn_readlane(k < 64 ? v[0] : k < 128 ? v[1] : k < 192 ? v[2] : v[3], k & 63);
    };
    const int64_t top = (int64_t)lo + 1 + (int64_t)m * step;
    if (m > 0) {
      lo = lo + 1 + (m - 1) * step;
      begin = probe(m - 1);
    }
    if (m < 256 && top < hi) {
      hi = (int)top;
      end = probe(m);
    }
  }
  return Span{lo, begin, end};
}

// Calls run(sample's span, first row, end) for the samples' parts of rows r0 .. r1 - 1, in
// order (uniform over the workgroup).
template <class Run>
__device__ inline void pieces_of(const GroupNormArgs& a, int64_t r0, int64_t r1, Run&& run) {
  int64_t r = r0;
  while (r < r1) {
    const Span s = span_of(a, r);
    if (s.s >= a.batch) return;
    const int64_t end = min(r1, max(s.end, r + 1));  // (offsets that decrease still end)
    if (s.s >= 0) run(s, r, end);
    r = end;
  }
}

// A thread's place among columns first .. first + width - 1 of whole groups: vector t of a
// row, row lane rl of rpb.
template <int V>
struct Place {
  int rl, rpb, col, skip, split, group[V];
  bool on;
  __device__ inline Place(int first, int width, int per, int nt) {
    const RowLane lane((int)threadIdx.x, (width + V - 1) / V, nt);
    rpb = lane.rpb;
    rl = lane.rl;
    on = lane.on;
    const int at = min(lane.t * V, width - V);
    col = first + at;
    skip = lane.t * V - at;
    split = min(V, ROW8_BLOCK - (col & (ROW8_BLOCK - 1)));
    group[0] = col / per;
    int left = per - (col - group[0] * per);  // columns of the group from here on
#pragma unroll
    for (int e = 1; e < V; ++e) {
      --left;
      group[e] = group[e - 1] + (left == 0 ? 1 : 0);
      left = left == 0 ? per : left;
    }
  }
};

// gain and shift of a thread's columns
template <int V>
struct Params {
  float gain[V], shift[V];
  __device__ inline Params(const GroupNormArgs& a, int col) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      gain[e] = a.gain ? a.gain[col + e] : 1.f;
      shift[e] = a.shift ? a.shift[col + e] : 0.f;
    }
  }
};

constexpr int FEW = 16;  // row lanes that one thread adds

// Sums over the row lanes of every column of the slice.  put() brings the threads' values
// together (uniform over the workgroup), col(c) is then the total of column c of the slice;
// `red` holds [rpb][width] floats and, for more than FEW row lanes, [FEW][width] behind them.
struct Totals {
  float* red;
  int width, rpb, nt;
  const float* from;
  int n;
  template <int V>
  __device__ inline void put(const Place<V>& p, int first, const float (&v)[V]) {
    __syncthreads();  // (the last totals have been read)
    if (p.on)
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (e >= p.skip) red[p.rl * width + p.col - first + e] = v[e];
    __syncthreads();
    from = red;
    n = rpb;
    if (rpb > FEW) {  // (then there are more threads than columns)
      const int parts = min(nt / width, FEW), q = threadIdx.x / width, c = threadIdx.x - q * width;
      float* to = red + rpb * width;
      if (q < parts) {
        float s = 0.f;
#pragma unroll 4
        for (int k = q; k < rpb; k += parts) s += red[k * width + c];
        to[q * width + c] = s;
      }
      __syncthreads();
      from = to;
      n = parts;
    }
  }
  __device__ inline float col(int c) const {
    float s = from[c];
#pragma unroll 4
    for (int k = 1; k < n; ++k) s += from[k * width + c];
    return s;
  }
};
// floats of `red`
__host__ __device__ inline int totals_floats(int rpb, int width) {
  return (rpb > 0 ? rpb : 1) * width + (rpb > FEW ? FEW * width : 0);
}

// done(group, sum of value(c) over its columns c, counted from the slice's first) for the
// `groups` groups of a slice, by the first of each group's lanes.
template <int L, class Value, class Done>
__device__ inline void group_totals_by(int groups, int per, Value&& value, Done&& done) {
  const int sub = threadIdx.x % L;
  for (int g = threadIdx.x / L; g < groups; g += blockDim.x / L) {
    float s = 0.f;
    for (int c = sub; c < per; c += L) s += value(g * per + c);
    if constexpr (L > 1) s = group_sum<L>(s);
    if (sub == 0) done(g, s);
  }
}
template <class Value, class Done>
__device__ inline void group_totals(int groups, int per, Value&& value, Done&& done) {
  if (per <= 4) group_totals_by<1>(groups, per, value, done);
  else if (per <= 64) group_totals_by<8>(groups, per, value, done);
  else group_totals_by<64>(groups, per, value, done);
}

// Sum of value(k) for k = first, first + step, .. below end, U at a time in flight (none of
// them alone behind the last whole group: a trip through memory for each would be most of
// a short sum's time).
template <int U, class Value>
__device__ inline float strided_sum(int first, int end, int step, Value&& value) {
  float s = 0.f;
  for (int k = first; k < end; k += U * step) {
    float v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = value(min(k + u * step, end - 1));
#pragma unroll
    for (int u = 0; u < U; ++u) s += k + u * step < end ? v[u] : 0.f;
  }
  return s;
}

// ---------------------------------------------------------------------------
// forward

__device__ inline void empty_stats(const GroupNormArgs& a, int64_t b) {
  for (int g = 0; g < a.groups; ++g) {
    a.stats[b * a.groups + g] = 0.f;
    a.stats[((int64_t)a.batch + b) * a.groups + g] = 1.f / sqrtf(a.eps);
  }
}

// Mean and 1 / deviation of group g of a sample out of its pieces, by L lanes of which this
// is number `lane`.
struct Stats {
  float mean, r;
};
template <int L>
__device__ inline Stats join_pieces(const GroupNormArgs& a, int64_t chunk, const Span& s, int g, int lane) {
  const int64_t lo = max(s.begin, (int64_t)0), hi = min(s.end, a.rows);
  if (lo >= hi) return Stats{0.f, 1.f / sqrtf(a.eps)};
  const int c0 = (int)(lo / chunk), pieces = (int)((hi - 1) / chunk) - c0 + 1;
  const float n = (float)(int)(hi - lo) * (float)a.per;
  const float* part = a.ws + ((int64_t)c0 + s.s) * 2 * a.groups + 2 * g;
  const int step = 2 * a.groups;
  auto rows = [&](int k) {
    const int64_t c = (c0 + k) * chunk;
    return (float)(int)(min(hi, c + chunk) - max(lo, c)) * (float)a.per;
  };
  const float mean =
      group_sum<L>(strided_sum<4>(lane, pieces, L, [&](int k) { return rows(k) * part[k * step]; })) / n;
  const float m2 = group_sum<L>(strided_sum<4>(lane, pieces, L, [&](int k) {
    const float d = part[k * step] - mean;
    return part[k * step + 1] + rows(k) * d * d;
  }));
  return Stats{mean, 1.f / sqrtf(m2 / n + a.eps)};
}

// First launch: mean and summed squares of deviations of every piece and group.  Bound by
// reading x: 589824 rows of 256 in bf16 (302 MB) 50 us; where rows are few, by the chain of load,
// sum and join: 200001 of 100 (40 MB) 13.  f32 rows of more than 1024 columns (1024 threads, 128
// registers each) send 58 registers through scratch memory: 20000 rows of 2048 forward 101 us with
// the last launch, bf16 57.
template <typename T, int V, int NT>
__global__ void __launch_bounds__(NT) k_group_norm_sums(GroupNormArgs a, int64_t chunk) {
  extern __shared__ float smem[];
  const Place<V> p(0, a.cols, a.per, NT);
  const int64_t c = blockIdx.x, r0 = c * chunk, r1 = min(a.rows, r0 + chunk);
  typedef Held<T, V, false> Q;
  typedef FromX<T, V, false> X;
  const Share whole((int)(r1 - r0), p.rl, p.rpb, p.on);
  const X first(a, r0 + whole.rl, p.col, p.split, p.rpb);
  Stream<Q, 8> rows;
  rows.fetch(first, 0, max(whole.n - 1, 0));
  Totals tot{smem, a.cols, p.rpb, NT};
  float* mean = smem + totals_floats(p.rpb, a.cols);  // [groups]
  if (a.begin)  // samples without rows have no piece
    for (int64_t b = c * NT + threadIdx.x; b < a.batch; b += (int64_t)gridDim.x * NT)
      if (a.begin[b] >= a.begin[b + 1]) empty_stats(a, b);
  pieces_of(a, r0, r1, [&](const Span& s, int64_t lo, int64_t hi) {
    const Share h((int)(hi - lo), p.rl, p.rpb, p.on);
    const X x(a, lo + h.rl, p.col, p.split, p.rpb);
    if (lo > r0) rows.fetch(x, 0, max(h.n - 1, 0));
    float pivot[V], s1[V], s2[V];
    rows.q[0].values(pivot, p.split);
#pragma unroll
    for (int e = 0; e < V; ++e) s1[e] = s2[e] = 0.f;
    rows.run(x, h, [&](const Q& q, int, auto valid) {
      float f[V];
      q.values(f, p.split);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = valid ? f[e] - pivot[e] : 0.f;
        s1[e] += d;
        s2[e] += d * d;
      }
    });
    const float n = (float)h.n, rn = h.n ? 1.f / n : 0.f, count = (float)(int)(hi - lo) * (float)a.per;
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = h.n ? s1[e] + n * pivot[e] : 0.f;
    tot.put(p, 0, v);
    group_totals(a.groups, a.per, [&](int col) { return tot.col(col); }, [&](int g, float sum) { mean[g] = sum / count; });
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float d = pivot[e] + s1[e] * rn - mean[p.group[e]];
      v[e] = h.n ? (s2[e] - s1[e] * s1[e] * rn) + n * d * d : 0.f;
    }
    tot.put(p, 0, v);
    float* out = a.ws + (c + s.s) * 2 * a.groups;
    group_totals(a.groups, a.per, [&](int col) { return tot.col(col); },
                 [&](int g, float sum) {
                   out[2 * g] = mean[g];
                   out[2 * g + 1] = sum;
                 });
  });
}

// Where samples have many pieces, a launch of its own: mean and 1 / deviation of every sample
// and group.
__global__ void __launch_bounds__(256) k_group_norm_stats(GroupNormArgs a, int64_t chunk) {
  const int64_t items = (int64_t)a.batch * a.groups;
  for (int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < items; i += (int64_t)gridDim.x * 4) {
    const int s = (int)(i / a.groups);
    const Stats v = join_pieces<64>(a, chunk, Span{s, sample_begin(a, s), sample_begin(a, s + 1)}, (int)(i - (int64_t)s * a.groups),
                                    threadIdx.x & 63);
    if ((threadIdx.x & 63) == 0) {
      a.stats[i] = v.mean;
      a.stats[items + i] = v.r;
    }
  }
}

// Last launch: the rows.  JOIN: the statistics come from the pieces, and the workgroup with
// a sample's first row stores them (a launch less where samples have few pieces).  Bound by
// memory: 589824 rows of 256 108 us, 5.6 TB/s with x partly from the last-level cache; 200001 of
// 100 14, latency again.
template <typename T, int V, int NT, bool SILU, bool JOIN>
__global__ void __launch_bounds__(NT) k_group_norm_rows(GroupNormArgs a, int64_t chunk) {
  extern __shared__ float smem[];  // JOIN: [2][groups]
  const Place<V> p(0, a.cols, a.per, NT);
  const int64_t c = (int64_t)gridDim.x - 1 - blockIdx.x, r0 = c * chunk, r1 = min(a.rows, r0 + chunk);
  typedef Held<T, V, false> Q;
  typedef FromX<T, V, false> X;
  const Share whole((int)(r1 - r0), p.rl, p.rpb, p.on);
  const X first(a, r0 + whole.rl, p.col, p.split, p.rpb);
  Stream<Q, 4> rows;
  rows.fetch(first, 0, max(whole.n - 1, 0));
  const Params<V> w(a, p.col);
  pieces_of(a, r0, r1, [&](const Span& s, int64_t lo, int64_t hi) {
    const Share h((int)(hi - lo), p.rl, p.rpb, p.on);
    const X x(a, lo + h.rl, p.col, p.split, p.rpb);
    if (lo > r0) rows.fetch(x, 0, max(h.n - 1, 0));
    const int64_t all = (int64_t)a.batch * a.groups, at = (int64_t)s.s * a.groups;
    float mean[V], r[V];
    if constexpr (JOIN) {
      __syncthreads();  // (the last piece's have been read)
      for (int g = threadIdx.x >> 3; g < a.groups; g += NT / 8) {
        const Stats v = join_pieces<8>(a, chunk, s, g, threadIdx.x & 7);
        if ((threadIdx.x & 7) == 0) {
          smem[g] = v.mean;
          smem[a.groups + g] = v.r;
          if (lo == s.begin) {
            a.stats[at + g] = v.mean;
            a.stats[all + at + g] = v.r;
          }
        }
      }
      __syncthreads();
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
      mean[e] = JOIN ? smem[p.group[e]] : a.stats[at + p.group[e]];
      r[e] = JOIN ? smem[a.groups + p.group[e]] : a.stats[all + at + p.group[e]];
    }
    const From<T, V> y(a.y, a.y_stride, lo + h.rl, p.col, p.rpb);
    rows.run(x, h, [&](const Q& q, int k, auto valid) {
      float f[V];
      q.values(f, p.split);
#pragma unroll
      for (int e = 0; e < V; ++e)
        f[e] = activated<SILU>(affine(normal(f[e], mean[e], r[e]), w.gain[e], w.shift[e]), a.slope);
      if (valid && p.on) store_pack<T, V>(y.put(k), f, p.skip, a.stream);
    });
  });
}

// Workgroups of the small kernels: samples s0, s0 + step, .. of a slice of `slice` groups.
struct Slice {
  int first, width, g0, groups, s0, step;
  __device__ inline Slice(const GroupNormArgs& a, int slice, int slices) {
    const int per = a.per;
    s0 = blockIdx.x / slices;
    const int k = blockIdx.x - s0 * slices;
    step = gridDim.x / slices;
    g0 = k * slice;
    groups = min(slice, a.groups - g0);
    first = g0 * per;
    width = groups * per;
  }
};

// Small samples: a thread's NV rows in registers, so that x is read once.  Bound by latency: one
// character (150 rows of 10, f32) 6.3 to 6.8 us, of which a launch is 2.4.  With 512 threads and
// bf16 the rows' float32 values do not fit: 92 registers go through scratch memory, and 100 samples
// of 300 rows of 100 take 40 us where f32, without, takes 21.
template <typename T, int V, int NT, int NV, bool SILU>
__global__ void __launch_bounds__(NT) k_group_norm_small(GroupNormArgs a, int slice, int slices) {
  extern __shared__ float smem[];
  const Slice b(a, slice, slices);
  const int per = a.per;
  const Place<V> p(b.first, b.width, per, NT);
  Totals tot{smem, b.width, p.rpb, NT};
  float* mean = smem + totals_floats(p.rpb, b.width);  // [groups], then 1 / deviation
  float* dev = mean + b.groups;
  const Params<V> w(a, p.col);
  typedef Held<T, V, false> Q;
  for (int s = b.s0; s < a.batch; s += b.step) {
    const int64_t lo = min(max(sample_begin(a, s), (int64_t)0), a.rows);
    const int64_t hi = max(lo, min(sample_begin(a, s + 1), a.rows));
    const Share h((int)(hi - lo), p.rl, p.rpb, p.on);
    const bool held = h.most <= NV;
    const FromX<T, V, false> x(a, lo + max(h.rl, 0), p.col, p.split, p.rpb);
    Q q[NV];
    if (held)
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i < h.n) x.load(q[i], i);
    // run(values, k) for this thread's rows
    auto rows = [&](auto&& run) {
      float f[V];
      if (held) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (i < h.n) {
            q[i].values(f, p.split);
            run(f, i);
          }
      } else {
        for (int k = 0; k < h.n; k += 8) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x.load(q[i], min(k + i, h.n - 1));
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (k + i < h.n) {
              q[i].values(f, p.split);
              run(f, k + i);
            }
        }
      }
    };
    const float count = (float)(int)(hi - lo) * (float)per;
    float v[V], m[V], r[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = 0.f;
    rows([&](const float(&f)[V], int) {
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] += f[e];
    });
    tot.put(p, b.first, v);
    group_totals(b.groups, per, [&](int c) { return tot.col(c); },
                 [&](int g, float sum) { mean[g] = hi > lo ? sum / count : 0.f; });
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) {
      m[e] = mean[p.group[e] - b.g0];
      v[e] = 0.f;
    }
    rows([&](const float(&f)[V], int) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = f[e] - m[e];
        v[e] += d * d;
      }
    });
    tot.put(p, b.first, v);
    group_totals(b.groups, per, [&](int c) { return tot.col(c); },
                 [&](int g, float sum) {
                   const float d = 1.f / sqrtf((hi > lo ? sum / count : 0.f) + a.eps);
                   dev[g] = d;
                   const int64_t at = (int64_t)s * a.groups + b.g0 + g;
                   a.stats[at] = mean[g];
                   a.stats[(int64_t)a.batch * a.groups + at] = d;
                 });
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) r[e] = dev[p.group[e] - b.g0];
    const From<T, V> y(a.y, a.y_stride, lo + max(h.rl, 0), p.col, p.rpb);
    rows([&](const float(&f)[V], int k) {
      float o[V];
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = activated<SILU>(affine(normal(f[e], m[e], r[e]), w.gain[e], w.shift[e]), a.slope);
      store_pack<T, V>(y.put(k), o, p.skip, a.stream);
    });
  }
}

// ---------------------------------------------------------------------------
// backward

template <typename T, int V, bool X8>
struct Pair {
  Held<T, V, X8> x;
  Pack<T, V> d;
  template <bool SILU>
  __device__ inline void values(const GroupNormArgs& a, const Place<V>& p, const Params<V>& w, const float (&mean)[V],
                                const float (&r)[V], float (&dz)[V], float (&h)[V]) const {
    x.values(h, p.split);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      h[e] = normal(h[e], mean[e], r[e]);
      dz[e] = gradient<SILU>(Elem<T>::to_f32(d.e[e]), h[e], w.gain[e], w.shift[e], a.slope);
    }
  }
};

template <typename T, int V, bool X8>
struct FromBoth {
  FromX<T, V, X8> x;
  From<T, V> d;
  __device__ inline FromBoth(const GroupNormArgs& a, int64_t row, const Place<V>& p)
      : x(a, row, p.col, p.split, p.rpb), d(a.dy, a.dy_stride, row, p.col, p.rpb) {}
  __device__ inline void load(Pair<T, V, X8>& q, int k) const {
    x.load(q.x, k);
    d.load(q.d, k);
  }
};

// r (dz gain - m1 - h m2) = dz (r gain) - r m1 - h (r m2), the products made once a thread
template <int V>
struct Slopes {
  float g[V], c1[V], c2[V];
};

// What the backward pass keeps in its workspace.
struct BwdParts {
  float* chunk;  // sums of dz h and of dz over a chunk's (a workgroup's) rows: [2][parts][cols]
  float* piece;  // [chunks + batch][2][cols]: of dz and of dz h over a piece's rows
  float* means;  // [2][batch][groups]: sum t / n, sum t h / n
};
__device__ inline BwdParts bwd_parts(const GroupNormArgs& a, int64_t parts) {
  BwdParts b;
  b.chunk = a.ws;
  b.piece = b.chunk + parts * 2 * a.cols;
  b.means = b.piece + (parts + a.batch) * 2 * a.cols;
  return b;
}

// First launch: a piece's sums of dz and dz h for every column, and a chunk's.  Bound by reading
// dy and x: 43 us where x is in 8 bits in rows of 512 and the next launch takes 68, 4.4 to 4.7 TB/s
// in both; by latency in smaller ones: 20011 rows of 300 in f32 16.5, one
// sample of 200001 rows of 100 in bf16 18.9.
template <typename T, int V, int NT, bool X8, bool SILU>
__global__ void __launch_bounds__(NT) k_group_norm_bwd_sums(GroupNormArgs a, int64_t chunk) {
  extern __shared__ float smem[];
  const Place<V> p(0, a.cols, a.per, NT);
  const int64_t c = blockIdx.x, r0 = c * chunk, r1 = min(a.rows, r0 + chunk);
  typedef Pair<T, V, X8> Q;
  typedef FromBoth<T, V, X8> X;
  const Share whole((int)(r1 - r0), p.rl, p.rpb, p.on);
  const X first(a, r0 + whole.rl, p);
  Stream<Q, 4> rows;
  rows.fetch(first, 0, max(whole.n - 1, 0));
  Totals tot{smem, a.cols, p.rpb, NT};
  float* total = smem + totals_floats(p.rpb, a.cols);  // [2][cols]
  const BwdParts parts = bwd_parts(a, gridDim.x);
  const Params<V> w(a, p.col);
  for (int i = threadIdx.x; i < 2 * a.cols; i += NT) total[i] = 0.f;
  pieces_of(a, r0, r1, [&](const Span& s, int64_t lo, int64_t hi) {
    const Share h((int)(hi - lo), p.rl, p.rpb, p.on);
    const X x(a, lo + h.rl, p);
    if (lo > r0) rows.fetch(x, 0, max(h.n - 1, 0));
    float mean[V], r[V], sum[2][V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int64_t at = (int64_t)s.s * a.groups + p.group[e];
      mean[e] = a.stats[at];
      r[e] = a.stats[(int64_t)a.batch * a.groups + at];
      sum[0][e] = sum[1][e] = 0.f;
    }
    rows.run(x, h, [&](const Q& q, int, auto valid) {
      float dz[V], h[V];
      q.template values<SILU>(a, p, w, mean, r, dz, h);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        sum[0][e] += valid ? dz[e] : 0.f;
        sum[1][e] += valid ? dz[e] * h[e] : 0.f;
      }
    });
    float* out = parts.piece + (c + s.s) * 2 * a.cols;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      tot.put(p, 0, sum[k]);
      for (int i = threadIdx.x; i < a.cols; i += NT) {  // (each column is one thread's)
        const float v = tot.col(i);
        out[k * a.cols + i] = v;
        total[k * a.cols + i] += v;
      }
    }
  });
  for (int i = threadIdx.x; i < a.cols; i += NT) {
    parts.chunk[c * a.cols + i] = total[a.cols + i];
    parts.chunk[((int64_t)gridDim.x + c) * a.cols + i] = total[i];
  }
}

// dgain (which = 0) and dshift: some columns' sums over the chunks, 64 lanes a column.
template <int NT>
__device__ inline void param_sums(const GroupNormArgs& a, const float* chunk, int parts, int block, float* smem) {
  constexpr int LANES = 64, COLS = NT / LANES;
  const int cb = (a.cols + COLS - 1) / COLS, which = block / cb;
  const int at = threadIdx.x % COLS, c = (block - which * cb) * COLS + at, sl = threadIdx.x / COLS;
  const float* p = chunk + (int64_t)which * parts * a.cols;
  float* out = which ? a.dshift : a.dgain;
  float v = c < a.cols ? strided_sum<16>(sl, parts, LANES, [&](int k) { return p[(int64_t)k * a.cols + c]; }) : 0.f;
  smem[sl * COLS + at] = v;
  __syncthreads();
  if (sl == 0 && c < a.cols && out) {
#pragma unroll 8
    for (int k = 1; k < LANES; ++k) v += smem[k * COLS + at];
    out[c] = v;
  }
}
template <int NT>
int param_blocks(int cols) {
  return 2 * ((cols + NT / 64 - 1) / (NT / 64));
}

__global__ void __launch_bounds__(1024) k_group_norm_params(GroupNormArgs a, int parts) {
  __shared__ float smem[1024];
  param_sums<1024>(a, a.ws, parts, blockIdx.x, smem);
}

// sum t / n and sum t h / n of a slice of a sample's groups, out of its pieces: done(k, group of
// the slice, value) with k = 0 for the first.  smem: [2][join_lanes(NT, width)][width].
template <int NT, class Done>
__device__ inline void join_means(const GroupNormArgs& a, const float* piece, int64_t chunk, const Span& s, int first,
                                  int groups, int per, float* smem, Done&& done) {
  const int64_t lo = max(s.begin, (int64_t)0), hi = min(s.end, a.rows);
  const int64_t c0 = lo / chunk;
  const int pieces = (int)((hi - 1) / chunk - c0) + 1, step = 2 * a.cols;
  const float rn = 1.f / ((float)(int)(hi - lo) * (float)per);
  const int width = groups * per, lanes = min(join_lanes(NT, width), pieces);
  __syncthreads();  // (what smem held has been read)
  for (int i = threadIdx.x; i < lanes * width; i += NT) {
    const int l = i / width, col = first + i - l * width;
    const float* q = piece + (c0 + s.s) * step + col;
    const float g = a.gain ? a.gain[col] : 1.f;
    float u = 0.f, v = 0.f;
    constexpr int U = NT == 1024 ? 16 : 8;
    for (int c = l; c < pieces; c += U * lanes) {
      float x[U], y[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int64_t at = (int64_t)min(c + k * lanes, pieces - 1) * step;
        x[k] = q[at];
        y[k] = q[at + a.cols];
      }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        u += c + k * lanes < pieces ? x[k] : 0.f;
        v += c + k * lanes < pieces ? y[k] : 0.f;
      }
    }
    smem[i] = u * g;
    smem[lanes * width + i] = v * g;
  }
  __syncthreads();
  // many lanes: eight of them first
  const int few = min(lanes, 8);
  if (lanes > few) {
    for (int i = threadIdx.x; i < 2 * few * width; i += NT) {
      const int l = i / width, c = i - l * width, k = l / few;
      float* p = smem + (k * lanes + l - k * few) * width + c;
      float v = p[0];
#pragma unroll 4
      for (int q = few; q < lanes - (l - k * few); q += few) v += p[q * width];
      p[0] = v;  // (this thread's alone)
    }
    __syncthreads();
  }
  for (int k = 0; k < 2; ++k)
    group_totals(groups, per,
                 [&](int c) {
                   float v = 0.f;
#pragma unroll 8
                   for (int l = 0; l < few; ++l) v += smem[(k * lanes + l) * width + c];
                   return v;
                 },
                 [&](int g, float sum) { done(k, g, sum * rn); });
}

// Where samples have many pieces, a launch of its own.  Its first `sample_blocks` workgroups: the means of
// t and t h over the samples and some of their groups; the others: the gain's and shift's
// gradients.
__global__ void __launch_bounds__(1024) k_group_norm_bwd_means(GroupNormArgs a, int64_t chunk, int chunks,
                                                               int sample_blocks, int slice) {
  extern __shared__ float smem[];
  const BwdParts parts = bwd_parts(a, chunks);
  if ((int)blockIdx.x >= sample_blocks) {
    param_sums<1024>(a, parts.chunk, chunks, (int)blockIdx.x - sample_blocks, smem);
    return;
  }
  const int per = a.per, slices = (a.groups + slice - 1) / slice;
  const int64_t items = (int64_t)a.batch * slices;
  for (int64_t item = blockIdx.x; item < items; item += sample_blocks) {
    const int s = (int)(item / slices), g0 = (int)(item - (int64_t)s * slices) * slice;
    const Span sp{s, sample_begin(a, s), sample_begin(a, s + 1)};
    if (max(sp.begin, (int64_t)0) >= min(sp.end, a.rows)) continue;
    join_means<1024>(a, parts.piece, chunk, sp, g0 * per, min(slice, a.groups - g0), per, smem,
                     [&](int k, int g, float v) { parts.means[((int64_t)k * a.batch + s) * a.groups + g0 + g] = v; });
  }
}

// Last launch: dx.  JOIN: the means come from the pieces, and the workgroups behind those of the
// chunks sum the gain's and shift's gradients.  Reads dy and x again and writes dx: 20011 rows
// of 300 in f32 24.7 us, one sample of 200001 of 100 in bf16 (means by a launch of their own,
// 10.2) 23.3.
template <typename T, int V, int NT, bool X8, bool SILU, bool JOIN>
__global__ void __launch_bounds__(NT) k_group_norm_bwd_rows(GroupNormArgs a, int64_t chunk, int chunks) {
  extern __shared__ float smem[];  // JOIN: join_floats, then [2][groups]
  const BwdParts parts = bwd_parts(a, chunks);
  const int per = a.per;
  float* joined = smem + join_floats(NT, a.cols);
  if (JOIN && (int)blockIdx.x >= chunks) {
    param_sums<NT>(a, parts.chunk, chunks, (int)blockIdx.x - chunks, smem);
    return;
  }
  const Place<V> p(0, a.cols, per, NT);
  const int64_t c = (int64_t)chunks - 1 - blockIdx.x, r0 = c * chunk, r1 = min(a.rows, r0 + chunk);
  typedef Pair<T, V, X8> Q;
  typedef FromBoth<T, V, X8> X;
  const Share whole((int)(r1 - r0), p.rl, p.rpb, p.on);
  const X ahead(a, r0 + whole.rl, p);
  Stream<Q, 4> rows;
  rows.fetch(ahead, 0, max(whole.n - 1, 0));
  const Params<V> w(a, p.col);
  pieces_of(a, r0, r1, [&](const Span& s, int64_t lo, int64_t hi) {
    const Share h((int)(hi - lo), p.rl, p.rpb, p.on);
    const X x(a, lo + h.rl, p);
    if (lo > r0) rows.fetch(x, 0, max(h.n - 1, 0));
    if constexpr (JOIN) {
      join_means<NT>(a, parts.piece, chunk, s, 0, a.groups, per, smem,
                     [&](int k, int g, float v) { joined[k * a.groups + g] = v; });
      __syncthreads();
    }
    float mean[V], r[V];
    Slopes<V> k;
    const int64_t all = (int64_t)a.batch * a.groups, at = (int64_t)s.s * a.groups;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      mean[e] = a.stats[at + p.group[e]];
      r[e] = a.stats[all + at + p.group[e]];
      k.g[e] = r[e] * w.gain[e];
      k.c1[e] = -r[e] * (JOIN ? joined[p.group[e]] : parts.means[at + p.group[e]]);
      k.c2[e] = -r[e] * (JOIN ? joined[a.groups + p.group[e]] : parts.means[all + at + p.group[e]]);
    }
    const From<T, V> dx(a.dx, a.dx_stride, lo + h.rl, p.col, p.rpb);
    rows.run(x, h, [&](const Q& q, int i, auto valid) {
      float dz[V], h[V];
      q.template values<SILU>(a, p, w, mean, r, dz, h);
#pragma unroll
      for (int e = 0; e < V; ++e) dz[e] = fmaf(dz[e], k.g[e], fmaf(h[e], k.c2[e], k.c1[e]));
      if (valid && p.on) store_pack<T, V>(dx.put(i), dz, p.skip, a.stream);
    });
  });
}

// Small samples: both rows in registers; a workgroup's sums of dz h and dz over its samples
// go to its row of the partial sums.
template <typename T, int V, int NT, int NV, bool X8, bool SILU>
__global__ void __launch_bounds__(NT) k_group_norm_bwd_small(GroupNormArgs a, int slice, int slices) {
  extern __shared__ float smem[];
  const Slice b(a, slice, slices);
  const int per = a.per;
  const Place<V> p(b.first, b.width, per, NT);
  Totals tot{smem, b.width, p.rpb, NT};
  float* total = smem + totals_floats(p.rpb, b.width);  // [2][width]
  float* mean = total + 2 * b.width;                     // [2][groups]
  const Params<V> w(a, p.col);
  typedef Pair<T, V, X8> Q;
  for (int i = threadIdx.x; i < 2 * b.width; i += NT) total[i] = 0.f;
  for (int s = b.s0; s < a.batch; s += b.step) {
    const int64_t lo = min(max(sample_begin(a, s), (int64_t)0), a.rows);
    const int64_t hi = max(lo, min(sample_begin(a, s + 1), a.rows));
    if (lo >= hi) continue;
    const Share h((int)(hi - lo), p.rl, p.rpb, p.on);
    const bool held = h.most <= NV;
    const FromBoth<T, V, X8> x(a, lo + h.rl, p);
    Q q[NV];
    if (held)
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i < h.n) x.load(q[i], i);
    float m[V], r[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int64_t at = (int64_t)s * a.groups + p.group[e];
      m[e] = a.stats[at];
      r[e] = a.stats[(int64_t)a.batch * a.groups + at];
    }
    // run(dz, h, k) for this thread's rows
    auto rows = [&](auto&& run) {
      float dz[V], hh[V];
      if (held) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (i < h.n) {
            q[i].template values<SILU>(a, p, w, m, r, dz, hh);
            run(dz, hh, i);
          }
      } else {
        for (int k = 0; k < h.n; k += 4) {
#pragma unroll
          for (int i = 0; i < 4; ++i) x.load(q[i], min(k + i, h.n - 1));
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (k + i < h.n) {
              q[i].template values<SILU>(a, p, w, m, r, dz, hh);
              run(dz, hh, k + i);
            }
        }
      }
    };
    float sum[2][V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[0][e] = sum[1][e] = 0.f;
    rows([&](const float(&dz)[V], const float(&h)[V], int) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        sum[0][e] += dz[e];
        sum[1][e] += dz[e] * h[e];
      }
    });
    const float rn = 1.f / ((float)(int)(hi - lo) * (float)per);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      tot.put(p, b.first, sum[k]);
      for (int i = threadIdx.x; i < b.width; i += NT) total[k * b.width + i] += tot.col(i);
      group_totals(b.groups, per, [&](int c) { return tot.col(c) * (a.gain ? a.gain[b.first + c] : 1.f); },
                   [&](int g, float v) { mean[k * b.groups + g] = v * rn; });
    }
    __syncthreads();
    Slopes<V> k;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      k.g[e] = r[e] * w.gain[e];
      k.c1[e] = -r[e] * mean[p.group[e] - b.g0];
      k.c2[e] = -r[e] * mean[b.groups + p.group[e] - b.g0];
    }
    const From<T, V> dx(a.dx, a.dx_stride, lo + h.rl, p.col, p.rpb);
    rows([&](const float(&dz)[V], const float(&h)[V], int i) {
      float o[V];
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = fmaf(dz[e], k.g[e], fmaf(h[e], k.c2[e], k.c1[e]));
      store_pack<T, V>(dx.put(i), o, p.skip, a.stream);
    });
  }
  for (int i = threadIdx.x; i < b.width; i += NT) {  // (each column is one thread's)
    a.ws[(int64_t)b.s0 * a.cols + b.first + i] = total[b.width + i];
    a.ws[((int64_t)b.step + b.s0) * a.cols + b.first + i] = total[i];
  }
}

// ---------------------------------------------------------------------------
// how work is dealt

// Small samples.
constexpr int SMALL_PARTS = 1024;  // workgroups of a slice
// rows of a thread in registers: 128 bytes of x, or 64 of x and 64 of dy, with 256 threads
constexpr int small_rows(int threads, bool bf16, bool backward) {
  return (threads == 256 ? 1 : 2) * (backward ? (bf16 ? 8 : 4) : 8);
}
constexpr int SLICE_BYTES = 64;
struct Small {
  bool on;
  int threads, slice, slices, parts, width;
};
Small small_of(bool bf16, int64_t rows, int32_t cols, int32_t groups, int32_t batch, bool backward) {
  Small s{};
  if (batch <= 0 || rows <= 0) return s;
  const int per = cols / groups, size = bf16 ? 2 : 4;
  // as many slices as make two workgroups a compute unit, of SLICE_BYTES at least, and the
  // last one, which may be narrower, of a vector
  const int most = std::max(1, std::min(groups, per * size * groups / SLICE_BYTES));
  for (int want = std::min(most, std::max(1, (512 + batch - 1) / batch));; --want) {
    s.slice = (groups + want - 1) / want;
    s.slices = (groups + s.slice - 1) / s.slice;
    if (s.slices == 1 || (groups - (s.slices - 1) * s.slice) * per >= norm_vec(bf16, cols, backward)) break;
  }
  s.width = s.slice * per;
  const int v = norm_vec(bf16, s.width, backward), nvec = (s.width + v - 1) / v;
  const double mean = (double)rows / batch;  // rows of a sample; the largest have several times as many
  if (nvec > 512) return s;
  s.threads = nvec <= 256 && 3.0 * mean <= 256 / nvec * small_rows(256, bf16, backward) ? 256 : 512;
  s.parts = std::min(batch, SMALL_PARTS);
  s.on = (batch == 1 ? 1.0 : 3.0) * mean <= s.threads / nvec * small_rows(s.threads, bf16, backward);
  return s;
}

int sum_lds(int rpb, int width, int extra) { return (totals_floats(rpb, width) + extra) * 4; }

// LDS of a small kernel, `columns` and `each` floats beside the totals for every column and
// group.  The last slice may be narrower than the others, and its rows be dealt to more lanes.
template <int V>
int small_lds(const Small& s, const GroupNormArgs& a, int columns, int each) {
  const int last = a.groups - (s.slices - 1) * s.slice, per = a.per;
  int most = 0;
  for (const int groups : {s.slice, last}) {
    const int width = groups * per;
    most = std::max(most, sum_lds(s.threads / ((width + V - 1) / V), width, columns * width + each * groups));
  }
  return most;
}

template <typename T, int V, int NT, bool SILU>
hipError_t forward_large(const GroupNormArgs& a, const NormDeal& d, hipStream_t st) {
  hipError_t e = hipSuccess;
  if (a.rows > 0) {
    hipLaunchKernelGGL((k_group_norm_sums<T, V, NT>), dim3(d.chunks), dim3(NT), sum_lds(d.rpb, a.cols, a.groups), st, a,
                       d.chunk);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (d.join) {
      hipLaunchKernelGGL((k_group_norm_rows<T, V, NT, SILU, true>), dim3(d.chunks), dim3(NT), 2 * a.groups * 4, st, a,
                         d.chunk);
      return hipGetLastError();
    }
  }
  const int64_t items = ((int64_t)a.batch * a.groups + 3) / 4;
  hipLaunchKernelGGL(k_group_norm_stats, dim3((unsigned)std::min<int64_t>(items, 4096)), dim3(256), 0, st, a, d.chunk);
  e = hipGetLastError();
  if (e != hipSuccess || a.rows <= 0) return e;
  hipLaunchKernelGGL((k_group_norm_rows<T, V, NT, SILU, false>), dim3(d.chunks), dim3(NT), 0, st, a, d.chunk);
  return hipGetLastError();
}

template <typename T, int V, int NT, bool SILU>
hipError_t forward_small(const GroupNormArgs& a, const Small& s, hipStream_t st) {
  constexpr auto kernel = k_group_norm_small<T, V, NT, small_rows(NT, sizeof(T) == 2, false), SILU>;
  const int lds = small_lds<V>(s, a, 0, 2);
  const hipError_t e = allow_lds<kernel>(lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3(s.parts * s.slices), dim3(NT), lds, st, a, s.slice, s.slices);
  return hipGetLastError();
}

template <typename T, bool SILU>
hipError_t forward(const GroupNormArgs& a, hipStream_t st) {
  constexpr bool bf16 = sizeof(T) == 2;
  constexpr int VE = bf16 ? 8 : 4, WIDE = bf16 ? 512 : 1024;
  if (a.batch <= 0) return hipSuccess;
  const Small s = small_of(bf16, a.rows, a.cols, a.groups, a.batch, false);
  if (s.on) {
    const bool scalar = s.width < VE;
    if (s.threads == 256) return scalar ? forward_small<T, 1, 256, SILU>(a, s, st) : forward_small<T, VE, 256, SILU>(a, s, st);
    return scalar ? forward_small<T, 1, 512, SILU>(a, s, st) : forward_small<T, VE, 512, SILU>(a, s, st);
  }
  const NormDeal d = norm_deal(bf16, a.rows, a.cols, a.batch, false);
  if (a.cols < VE) return forward_large<T, 1, 256, SILU>(a, d, st);
  return d.threads == 256 ? forward_large<T, VE, 256, SILU>(a, d, st) : forward_large<T, VE, WIDE, SILU>(a, d, st);
}

template <typename T, int V, int NT, bool X8, bool SILU>
hipError_t backward_large(const GroupNormArgs& a, const NormDeal& d, hipStream_t st) {
  hipLaunchKernelGGL((k_group_norm_bwd_sums<T, V, NT, X8, SILU>), dim3(d.chunks), dim3(NT),
                     sum_lds(d.rpb, a.cols, 2 * a.cols), st, a, d.chunk);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (d.join) {
    constexpr auto kernel = k_group_norm_bwd_rows<T, V, NT, X8, SILU, true>;
    const int lds = std::max(NT, join_floats(NT, a.cols) + 2 * a.groups) * 4;
    e = allow_lds<kernel>(lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(d.chunks + param_blocks<NT>(a.cols)), dim3(NT), lds, st, a, d.chunk, d.chunks);
    return hipGetLastError();
  }
  const NormMeans m = norm_means(a.batch, a.groups, a.per);
  hipLaunchKernelGGL(k_group_norm_bwd_means, dim3((unsigned)(m.blocks + param_blocks<1024>(a.cols))), dim3(1024),
                     m.floats * 4, st, a, d.chunk, d.chunks, m.blocks, m.slice);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_group_norm_bwd_rows<T, V, NT, X8, SILU, false>), dim3(d.chunks), dim3(NT), 0, st, a, d.chunk,
                     d.chunks);
  return hipGetLastError();
}

template <typename T, int V, int NT, bool X8, bool SILU>
hipError_t backward_small(const GroupNormArgs& a, const Small& s, hipStream_t st) {
  constexpr auto kernel = k_group_norm_bwd_small<T, V, NT, small_rows(NT, sizeof(T) == 2, true), X8, SILU>;
  const int lds = small_lds<V>(s, a, 2, 2);
  hipError_t e = allow_lds<kernel>(lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3(s.parts * s.slices), dim3(NT), lds, st, a, s.slice, s.slices);
  e = hipGetLastError();
  if (e != hipSuccess || (!a.dgain && !a.dshift)) return e;
  hipLaunchKernelGGL(k_group_norm_params, dim3(param_blocks<1024>(a.cols)), dim3(1024), 0, st, a, s.parts);
  return hipGetLastError();
}

template <typename T, bool X8, bool SILU>
hipError_t backward(const GroupNormArgs& a, hipStream_t st) {
  constexpr bool bf16 = sizeof(T) == 2;
  const Small s = small_of(bf16, a.rows, a.cols, a.groups, a.batch, true);
  if (s.on) {
    const bool scalar = s.width < 4;
    if (s.threads == 256)
      return scalar ? backward_small<T, 1, 256, X8, SILU>(a, s, st) : backward_small<T, 4, 256, X8, SILU>(a, s, st);
    return scalar ? backward_small<T, 1, 512, X8, SILU>(a, s, st) : backward_small<T, 4, 512, X8, SILU>(a, s, st);
  }
  const NormDeal d = norm_deal(bf16, a.rows, a.cols, a.batch, true);
  if (a.cols < 4) return backward_large<T, 1, 256, X8, SILU>(a, d, st);
  return d.threads == 256 ? backward_large<T, 4, 256, X8, SILU>(a, d, st) : backward_large<T, 4, 1024, X8, SILU>(a, d, st);
}

}  // namespace

// Either way of dealing: which one a call takes may differ with its rows.
size_t group_norm_workspace(bool bf16, int64_t rows, int32_t cols, int32_t groups, int32_t batch, bool backward) {
  if (rows <= 0) return 0;
  const NormDeal d = norm_deal(bf16, rows, cols, batch, backward);
  const size_t pieces = (size_t)d.most + (size_t)batch;
  if (!backward) return pieces * 2 * (size_t)groups * 4;
  const size_t large = ((pieces + (size_t)d.most) * 2 * (size_t)cols + 2 * (size_t)batch * (size_t)groups) * 4;
  return std::max(large, (size_t)std::min(batch, SMALL_PARTS) * 2 * (size_t)cols * 4);
}

hipError_t launch_group_norm(bool bf16, const GroupNormArgs& a, hipStream_t st) {
  if (bf16) return a.silu ? forward<__bf16, true>(a, st) : forward<__bf16, false>(a, st);
  return a.silu ? forward<float, true>(a, st) : forward<float, false>(a, st);
}

hipError_t launch_group_norm_bwd(bool bf16, const GroupNormArgs& a, hipStream_t st) {
  if (a.rows <= 0 || a.batch <= 0) {  // sums over nothing
    const hipError_t e = a.dgain ? launch_fill_zero(a.dgain, (int64_t)a.cols * 4, st) : hipSuccess;
    return e == hipSuccess && a.dshift ? launch_fill_zero(a.dshift, (int64_t)a.cols * 4, st) : e;
  }
  if (a.codes) {
    if (bf16) return a.silu ? backward<__bf16, true, true>(a, st) : backward<__bf16, true, false>(a, st);
    return a.silu ? backward<float, true, true>(a, st) : backward<float, true, false>(a, st);
  }
  if (bf16) return a.silu ? backward<__bf16, false, true>(a, st) : backward<__bf16, false, false>(a, st);
  return a.silu ? backward<float, false, true>(a, st) : backward<float, false, false>(a, st);
}

}  // namespace sscn
