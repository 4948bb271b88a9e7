// Normalisation over the rows of a sample and the channels of a group, with an
// activation, forward and backward; rows are sites, channels last.
//
//   mean = sum x / n,  r = 1 / sqrt(sum (x - mean)^2 / n + eps)   over a sample and group
//   h = (x - mean) r,  z = h gain + shift,  y = act(z)
//   backward  dz = dy act'(z), t = dz gain, dx = r (t - sum t / n - h sum(t h) / n),
//             dgain = sum over rows of dz h, dshift = sum over rows of dz
//
// Memory-bound.  Samples are runs of rows of any lengths, known on the device only, so
// work is dealt by equal chunks of rows: a workgroup walks through the samples that its
// chunk meets.  The part of sample s in chunk c is piece c + s, which numbers all pieces
// without a scan.  Three launches: sums of each piece, sums of each sample, the result.
// The last one goes through the chunks backwards, so that it finds in the last-level cache
// what the first one read last.
//
// A thread owns one vector of V columns and every rpb-th row.  The last vector starts V
// columns before the row's end, where its first `skip` columns repeat those of the vector
// before (left out of every sum and not stored).  Variances: a thread
// sums deviations from its own first value of a column, which cannot cancel by more than
// the number of its rows, and threads, pieces and columns are joined by their means.
// Every sum is taken in an order that sizes alone decide.  All arithmetic is float32.

#include "common.h"
#include "kernels.h"
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
__device__ inline void store_pack(T* p, const float (&f)[V], int skip) {
  Pack<T, V> v;
#pragma unroll
  for (int e = 0; e < V; ++e) v.e[e] = Elem<T>::from_f32(f[e]);
  if (skip == 0) {
    __builtin_memcpy(p, &v, sizeof(v));
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
  __device__ inline void load(const GroupNormArgs& a, int64_t r, int col, int) {
    v = load_pack<T, V>((const T*)a.x + r * a.x_stride + col);
  }
  __device__ inline void values(float (&f)[V], int) const {
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = Elem<T>::to_f32(v.e[e]);
  }
};
template <typename T, int V>
struct Held<T, V, true> {
  uint8_t c[V], s0, s1;
  // split: elements before the next scale's block
  __device__ inline void load(const GroupNormArgs& a, int64_t r, int col, int split) {
    __builtin_memcpy(c, a.codes + r * row8_code_stride(a.cols) + col, V);
    const uint8_t* s = a.scales + r * row8_scale_stride(a.cols) + (col >> 7);
    s0 = s[0];
    s1 = split < V ? s[1] : s0;
  }
  __device__ inline void values(float (&f)[V], int split) const {
    if constexpr (V >= 4) {
#pragma unroll
      for (int q = 0; q < V; q += 4) {
        uint32_t w;
        __builtin_memcpy(&w, c + q, 4);
        row8_values4(w, 1.f, f + q);
      }
    } else {
      float t[4];
      row8_values4(c[0], 1.f, t);
      f[0] = t[0];
    }
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] *= row8_pow2(e < split ? s0 : s1);
  }
};

// z, every operation rounded by itself: forward and backward take the same branch of the
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
__device__ inline float activated(float z, float slope, bool silu) {
  if (silu) return z * sigmoid(z);
  return z < 0.f ? (slope == 0.f ? 0.f : slope * z) : z;
}
// The framework's rule at zero: a rectifier's derivative is 0 there, the leaky one's 1.
__device__ inline float slope_at(float z, float slope, bool silu) {
  if (silu) {
    const float s = sigmoid(z);
    return s * (1.f + z * (1.f - s));
  }
  return (slope == 0.f ? z > 0.f : z >= 0.f) ? 1.f : slope;
}

// The last sample that starts at row r or before it (-1: none; batch: r lies behind the
// last one), by a whole wave, 64 probes at a time.  Bounds hold for any offsets.
__device__ inline int sample_of(const GroupNormArgs& a, int64_t r) {
  if (!a.begin) return (int)(r / a.span);
  int lo = -1, hi = a.batch + 1;
  while (hi - lo > 1) {
    const int step = (hi - lo - 1 + 63) / 64;
    const int64_t at = (int64_t)lo + 1 + (int64_t)(threadIdx.x & 63) * step;
    const int m = __popcll(__ballot(at < hi && a.begin[at < hi ? at : 0] <= r));
    const int64_t top = (int64_t)lo + 1 + (int64_t)m * step;
    if (m > 0) lo = lo + 1 + (m - 1) * step;
    if (top < hi) hi = (int)top;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}
__device__ inline int64_t sample_begin(const GroupNormArgs& a, int s) { return a.begin ? a.begin[s] : s * a.span; }

// Calls run(sample, first row, end) for the samples' parts of rows r0 .. r1 - 1, in order
// (uniform over the workgroup).
template <class Run>
__device__ inline void pieces_of(const GroupNormArgs& a, int64_t r0, int64_t r1, Run&& run) {
  int64_t r = r0;
  while (r < r1) {
    const int s = sample_of(a, r);
    if (s >= a.batch) return;
    const int64_t next = sample_begin(a, s + 1);
    const int64_t end = min(r1, max(next, r + 1));  // (offsets that decrease still end)
    if (s >= 0) run(s, r, end);
    r = end;
  }
}

// A thread's place: vector t of the row, row lane rl of rpb.
template <int V>
struct Place {
  int t, rl, rpb, col, skip, split, group[V];
  bool on;
  __device__ inline Place(int cols, int groups, int nt) {
    const int nvec = (cols + V - 1) / V;
    rpb = nt / nvec;
    t = threadIdx.x % nvec;
    rl = threadIdx.x / nvec;
    on = rl < rpb;
    const int at = t * V;
    col = min(at, cols - V);
    skip = at - col;
    split = min(V, ROW8_BLOCK - (col & (ROW8_BLOCK - 1)));
    const int per = cols / groups;
#pragma unroll
    for (int e = 0; e < V; ++e) group[e] = (col + e) / per;
  }
};

// Sums over the row lanes of every column: red is [rpb][cols], the totals are in its first row.
template <int V>
__device__ inline void column_totals(const Place<V>& p, float* red, int cols, const float (&v)[V]) {
  __syncthreads();  // (the last totals have been read)
  if (p.on)
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e >= p.skip) red[p.rl * cols + p.col + e] = v[e];
  __syncthreads();
  for (int c = threadIdx.x; c < cols; c += blockDim.x) {
    float s = 0.f;
    for (int k = 0; k < p.rpb; ++k) s += red[k * cols + c];
    red[c] = s;
  }
  __syncthreads();
}

// lanes that share a group's sum
__device__ inline int lanes_of(int per) { return per <= 4 ? 1 : per <= 64 ? 8 : 64; }

// done(group, sum over its channels c of value(c)), by the first lane of each group's lanes.
template <class Value, class Done>
__device__ inline void group_totals(int first, int end, int per, Value&& value, Done&& done) {
  const int L = lanes_of(per), sub = threadIdx.x % L;
  for (int g = first + threadIdx.x / L; g < end; g += blockDim.x / L) {
    float s = 0.f;
    for (int c = sub; c < per; c += L) s += value(g * per + c);
    for (int d = 1; d < L; d *= 2) s += __shfl_xor(s, d);
    if (sub == 0) done(g, s);
  }
}

// Forward, first launch: mean and summed squares of deviations of every piece and group.
template <typename T, int V>
__global__ void __launch_bounds__(1024) k_group_norm_sums(GroupNormArgs a, int64_t chunk) {
  extern __shared__ float smem[];
  const Place<V> p(a.cols, a.groups, blockDim.x);
  float* red = smem;                          // [rpb][cols]
  float* mean = smem + max(p.rpb, 1) * a.cols;  // [groups]
  const int per = a.cols / a.groups;
  const int64_t c = blockIdx.x, r0 = c * chunk, r1 = min(a.rows, r0 + chunk);
  pieces_of(a, r0, r1, [&](int s, int64_t lo, int64_t hi) {
    float pivot[V], s1[V], s2[V];
#pragma unroll
    for (int e = 0; e < V; ++e) pivot[e] = s1[e] = s2[e] = 0.f;
    int n = 0;
    if (p.on && lo + p.rl < hi) {
      Held<T, V, false> x;
      x.load(a, lo + p.rl, p.col, p.split);
      x.values(pivot, p.split);
      n = (int)((hi - lo - p.rl + p.rpb - 1) / p.rpb);
      constexpr int U = 4;
      int i = 1;
      for (; i + U <= n; i += U) {
        Held<T, V, false> q[U];
#pragma unroll
        for (int u = 0; u < U; ++u) q[u].load(a, lo + p.rl + (int64_t)(i + u) * p.rpb, p.col, p.split);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float f[V];
          q[u].values(f, p.split);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float d = f[e] - pivot[e];
            s1[e] += d;
            s2[e] += d * d;
          }
        }
      }
      for (; i < n; ++i) {
        float f[V];
        x.load(a, lo + p.rl + (int64_t)i * p.rpb, p.col, p.split);
        x.values(f, p.split);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = f[e] - pivot[e];
          s1[e] += d;
          s2[e] += d * d;
        }
      }
    }
    const float rn = n ? 1.f / (float)n : 0.f, count = (float)(hi - lo) * (float)per;
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = s1[e] + (float)n * pivot[e];
    column_totals<V>(p, red, a.cols, v);
    group_totals(0, a.groups, per, [&](int col) { return red[col]; }, [&](int g, float sum) { mean[g] = sum / count; });
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float d = pivot[e] + s1[e] * rn - mean[p.group[e]];
      v[e] = n ? (s2[e] - s1[e] * s1[e] * rn) + (float)n * d * d : 0.f;
    }
    column_totals<V>(p, red, a.cols, v);
    float* out = a.ws + (c + s) * 2 * a.groups;
    group_totals(0, a.groups, per, [&](int col) { return red[col]; },
                 [&](int g, float sum) {
                   out[2 * g] = mean[g];
                   out[2 * g + 1] = sum;
                 });
  });
}

// Second launch: mean and 1 / deviation of every sample and group out of its pieces.
__global__ void __launch_bounds__(256) k_group_norm_stats(GroupNormArgs a, int64_t chunk) {
  const int per = a.cols / a.groups, lane = threadIdx.x & 63;
  const int64_t items = (int64_t)a.batch * a.groups;
  for (int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < items; i += (int64_t)gridDim.x * 4) {
    const int s = (int)(i / a.groups), g = (int)(i - (int64_t)s * a.groups);
    const int64_t lo = min(max(sample_begin(a, s), (int64_t)0), a.rows), hi = min(sample_begin(a, s + 1), a.rows);
    float mean = 0.f, m2 = 0.f;
    const float n = (float)max(hi - lo, (int64_t)0) * (float)per;
    if (lo < hi) {
      const int64_t c0 = lo / chunk, c1 = (hi - 1) / chunk;
      const float* part = a.ws + (int64_t)s * 2 * a.groups + 2 * g;
      auto rows = [&](int64_t c) { return (float)(min(hi, (c + 1) * chunk) - max(lo, c * chunk)) * (float)per; };
      float sum = 0.f;
      for (int64_t c = c0 + lane; c <= c1; c += 64) sum += rows(c) * part[c * 2 * a.groups];
      for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
      mean = sum / n;
      for (int64_t c = c0 + lane; c <= c1; c += 64) {
        const float d = part[c * 2 * a.groups] - mean;
        m2 += part[c * 2 * a.groups + 1] + rows(c) * d * d;
      }
      for (int d = 1; d < 64; d *= 2) m2 += __shfl_xor(m2, d);
      m2 /= n;
    }
    if (lane == 0) {
      a.stats[i] = mean;
      a.stats[items + i] = 1.f / sqrtf(m2 + a.eps);
    }
  }
}

// Third launch: the rows.
template <typename T, int V>
__global__ void __launch_bounds__(1024) k_group_norm_rows(GroupNormArgs a, int64_t chunk) {
  const Place<V> p(a.cols, a.groups, blockDim.x);
  const int64_t c = (int64_t)gridDim.x - 1 - blockIdx.x, r0 = c * chunk, r1 = min(a.rows, r0 + chunk);
  float gain[V], shift[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    gain[e] = a.gain ? a.gain[p.col + e] : 1.f;
    shift[e] = a.shift ? a.shift[p.col + e] : 0.f;
  }
  pieces_of(a, r0, r1, [&](int s, int64_t lo, int64_t hi) {
    float mean[V], r[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int64_t at = (int64_t)s * a.groups + p.group[e];
      mean[e] = a.stats[at];
      r[e] = a.stats[(int64_t)a.batch * a.groups + at];
    }
    if (!p.on) return;
    auto put = [&](const Held<T, V, false>& x, int64_t row) {
      float f[V];
      x.values(f, p.split);
#pragma unroll
      for (int e = 0; e < V; ++e)
        f[e] = activated(affine(normal(f[e], mean[e], r[e]), gain[e], shift[e]), a.slope, a.silu);
      store_pack<T, V>((T*)a.y + row * a.y_stride + p.col, f, p.skip);
    };
    constexpr int U = 4;
    int64_t row = lo + p.rl;
    for (; row + (U - 1) * p.rpb < hi; row += U * p.rpb) {
      Held<T, V, false> q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) q[u].load(a, row + u * p.rpb, p.col, p.split);
#pragma unroll
      for (int u = 0; u < U; ++u) put(q[u], row + u * p.rpb);
    }
    for (; row < hi; row += p.rpb) {
      Held<T, V, false> q;
      q.load(a, row, p.col, p.split);
      put(q, row);
    }
  });
}

// dz and h of a thread's vector.
template <typename T, int V, bool X8>
struct Gradient {
  Held<T, V, X8> x;
  Pack<T, V> d;
  __device__ inline void load(const GroupNormArgs& a, int64_t row, const Place<V>& p) {
    x.load(a, row, p.col, p.split);
    d = load_pack<T, V>((const T*)a.dy + row * a.dy_stride + p.col);
  }
  __device__ inline void values(const GroupNormArgs& a, const Place<V>& p, const float (&mean)[V], const float (&r)[V],
                                const float (&gain)[V], const float (&shift)[V], float (&dz)[V], float (&h)[V]) const {
    x.values(h, p.split);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      h[e] = normal(h[e], mean[e], r[e]);
      dz[e] = Elem<T>::to_f32(d.e[e]) * slope_at(affine(h[e], gain[e], shift[e]), a.slope, a.silu);
    }
  }
};

// What the backward pass keeps in its workspace.
struct BwdParts {
  float* piece;  // [chunks + batch][2][cols]: sums of dz and of dz h over a piece's rows
  float* chunk;  // the same over a chunk's rows: [2][chunks][cols], dz h first
  float* means;  // [2][batch][groups]: sum t / n, sum t h / n
};
__device__ inline BwdParts bwd_parts(const GroupNormArgs& a, int64_t chunks) {
  BwdParts b;
  b.piece = a.ws;
  b.chunk = b.piece + (chunks + a.batch) * 2 * a.cols;
  b.means = b.chunk + chunks * 2 * a.cols;
  return b;
}

// Backward, first launch: a piece's sums of dz and dz h for every column, and a chunk's.
template <typename T, int V, bool X8>
__global__ void __launch_bounds__(1024) k_group_norm_bwd_sums(GroupNormArgs a, int64_t chunk) {
  extern __shared__ float smem[];
  const Place<V> p(a.cols, a.groups, blockDim.x);
  float* red = smem;                           // [rpb][cols]
  float* total = smem + max(p.rpb, 1) * a.cols;  // [2][cols]
  const int64_t c = blockIdx.x, r0 = c * chunk, r1 = min(a.rows, r0 + chunk);
  const BwdParts parts = bwd_parts(a, gridDim.x);
  float gain[V], shift[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    gain[e] = a.gain ? a.gain[p.col + e] : 1.f;
    shift[e] = a.shift ? a.shift[p.col + e] : 0.f;
  }
  for (int i = threadIdx.x; i < 2 * a.cols; i += blockDim.x) total[i] = 0.f;
  pieces_of(a, r0, r1, [&](int s, int64_t lo, int64_t hi) {
    float mean[V], r[V], sum[2][V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int64_t at = (int64_t)s * a.groups + p.group[e];
      mean[e] = a.stats[at];
      r[e] = a.stats[(int64_t)a.batch * a.groups + at];
      sum[0][e] = sum[1][e] = 0.f;
    }
    if (p.on) {
      auto add = [&](const Gradient<T, V, X8>& q) {
        float dz[V], h[V];
        q.values(a, p, mean, r, gain, shift, dz, h);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          sum[0][e] += dz[e];
          sum[1][e] += dz[e] * h[e];
        }
      };
      constexpr int U = 4;
      int64_t row = lo + p.rl;
      for (; row + (U - 1) * p.rpb < hi; row += U * p.rpb) {
        Gradient<T, V, X8> q[U];
#pragma unroll
        for (int u = 0; u < U; ++u) q[u].load(a, row + u * p.rpb, p);
#pragma unroll
        for (int u = 0; u < U; ++u) add(q[u]);
      }
      for (; row < hi; row += p.rpb) {
        Gradient<T, V, X8> q;
        q.load(a, row, p);
        add(q);
      }
    }
    float* out = parts.piece + (c + s) * 2 * a.cols;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      column_totals<V>(p, red, a.cols, sum[k]);
      for (int i = threadIdx.x; i < a.cols; i += blockDim.x) {
        out[k * a.cols + i] = red[i];
        total[k * a.cols + i] += red[i];  // (each column is one thread's)
      }
    }
  });
  for (int i = threadIdx.x; i < a.cols; i += blockDim.x) {
    parts.chunk[c * a.cols + i] = total[a.cols + i];
    parts.chunk[((int64_t)gridDim.x + c) * a.cols + i] = total[i];
  }
}

constexpr int BWD_COLS = 64;  // columns of a workgroup of the second launch

// Second launch.  Its first `sample_blocks` workgroups: the means of t and t h over the
// samples and some of their groups; the others: the gain's and shift's gradients, 64
// columns each, in 16 interleaved slices of the chunks.
__global__ void __launch_bounds__(1024) k_group_norm_bwd_means(GroupNormArgs a, int64_t chunk, int chunks,
                                                               int sample_blocks, int slice) {
  extern __shared__ float smem[];
  const BwdParts parts = bwd_parts(a, chunks);
  const int per = a.cols / a.groups;
  if ((int)blockIdx.x >= sample_blocks) {
    const int b = (int)blockIdx.x - sample_blocks, cb = (a.cols + 63) / 64, which = b / cb;
    const int c = (b - which * cb) * 64 + (threadIdx.x & 63), sl = threadIdx.x >> 6;
    const float* p = parts.chunk + (int64_t)which * chunks * a.cols;
    float* out = which ? a.dshift : a.dgain;
    float v = 0.f;
    if (c < a.cols)
#pragma unroll 16
      for (int k = sl; k < chunks; k += 16) v += p[(int64_t)k * a.cols + c];
    smem[sl * 64 + (threadIdx.x & 63)] = v;
    __syncthreads();
    if (sl == 0 && c < a.cols && out) {
      for (int k = 1; k < 16; ++k) v += smem[k * 64 + threadIdx.x];
      out[c] = v;
    }
    return;
  }
  const int slices = (a.groups + slice - 1) / slice;
  const int64_t items = (int64_t)a.batch * slices;
  for (int64_t item = blockIdx.x; item < items; item += sample_blocks) {
    const int s = (int)(item / slices), g0 = (int)(item - (int64_t)s * slices) * slice;
    const int g1 = min(g0 + slice, a.groups), first = g0 * per, width = (g1 - g0) * per;
    const int64_t lo = min(max(sample_begin(a, s), (int64_t)0), a.rows), hi = min(sample_begin(a, s + 1), a.rows);
    if (lo >= hi) continue;
    const int64_t c0 = lo / chunk, c1 = (hi - 1) / chunk;
    const float rn = 1.f / ((float)(hi - lo) * (float)per);
    const int lanes = max(1, (int)blockDim.x / width);  // smem: [lanes][width], the totals first
    for (int k = 0; k < 2; ++k) {
      __syncthreads();
      for (int i = threadIdx.x; i < lanes * width; i += blockDim.x) {
        const int l = i / width, col = first + i - l * width;
        float v = 0.f;
        const float* q = parts.piece + (int64_t)s * 2 * a.cols + k * a.cols + col;
#pragma unroll 8
        for (int64_t c = c0 + l; c <= c1; c += lanes) v += q[c * 2 * a.cols];
        smem[i] = v * (a.gain ? a.gain[col] : 1.f);
      }
      __syncthreads();
      for (int i = threadIdx.x; i < width; i += blockDim.x) {
        float v = smem[i];
        for (int l = 1; l < lanes; ++l) v += smem[l * width + i];
        smem[i] = v;
      }
      __syncthreads();
      group_totals(g0, g1, per, [&](int col) { return smem[col - first]; },
                   [&](int g, float sum) { parts.means[((int64_t)k * a.batch + s) * a.groups + g] = sum * rn; });
    }
  }
}

// Third launch: dx.
template <typename T, int V, bool X8>
__global__ void __launch_bounds__(1024) k_group_norm_bwd_rows(GroupNormArgs a, int64_t chunk) {
  const Place<V> p(a.cols, a.groups, blockDim.x);
  const int64_t c = (int64_t)gridDim.x - 1 - blockIdx.x, r0 = c * chunk, r1 = min(a.rows, r0 + chunk);
  const BwdParts parts = bwd_parts(a, gridDim.x);
  float gain[V], shift[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    gain[e] = a.gain ? a.gain[p.col + e] : 1.f;
    shift[e] = a.shift ? a.shift[p.col + e] : 0.f;
  }
  pieces_of(a, r0, r1, [&](int s, int64_t lo, int64_t hi) {
    float mean[V], r[V], m1[V], m2[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int64_t at = (int64_t)s * a.groups + p.group[e], all = (int64_t)a.batch * a.groups;
      mean[e] = a.stats[at];
      r[e] = a.stats[all + at];
      m1[e] = parts.means[at];
      m2[e] = parts.means[all + at];
    }
    if (!p.on) return;
    auto put = [&](const Gradient<T, V, X8>& q, int64_t row) {
      float dz[V], h[V];
      q.values(a, p, mean, r, gain, shift, dz, h);
#pragma unroll
      for (int e = 0; e < V; ++e) dz[e] = r[e] * (dz[e] * gain[e] - m1[e] - h[e] * m2[e]);
      store_pack<T, V>((T*)a.dx + row * a.dx_stride + p.col, dz, p.skip);
    };
    constexpr int U = 2;
    int64_t row = lo + p.rl;
    for (; row + (U - 1) * p.rpb < hi; row += U * p.rpb) {
      Gradient<T, V, X8> q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) q[u].load(a, row + u * p.rpb, p);
#pragma unroll
      for (int u = 0; u < U; ++u) put(q[u], row + u * p.rpb);
    }
    for (; row < hi; row += p.rpb) {
      Gradient<T, V, X8> q;
      q.load(a, row, p);
      put(q, row);
    }
  });
}

struct Deal {
  int threads, rpb;
  int64_t chunk;
  int chunks, most;  // and a bound on them that grows with the rows
};

Deal deal(bool bf16, int64_t rows, int32_t cols) {
  const int ve = bf16 ? 8 : 4, v = cols < ve ? 1 : ve, nvec = (cols + v - 1) / v;
  Deal d;
  d.threads = nvec <= 256 ? 256 : nvec <= 512 ? 512 : 1024;
  d.rpb = d.threads / nvec;
  const int64_t most = 1024 * 256 / d.threads;  // workgroups that the compute units hold at once, or twice as many
  const int64_t least = 8 * d.rpb;              // rows that pay for a workgroup's sums
  d.chunk = std::max(least, (rows + most - 1) / most);
  d.chunks = (int)((rows + d.chunk - 1) / d.chunk);
  d.most = (int)std::min(most, (rows + least - 1) / least);
  return d;
}

int sum_lds(const Deal& d, int32_t cols, int extra) { return (std::max(d.rpb, 1) * cols + extra) * 4; }

template <typename T, int V>
hipError_t forward(const GroupNormArgs& a, hipStream_t st) {
  if (a.batch <= 0) return hipSuccess;
  const Deal d = deal(sizeof(T) == 2, a.rows, a.cols);
  hipError_t e = hipSuccess;
  if (a.rows > 0) {
    hipLaunchKernelGGL((k_group_norm_sums<T, V>), dim3(d.chunks), dim3(d.threads), sum_lds(d, a.cols, a.groups), st, a,
                       d.chunk);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int64_t items = ((int64_t)a.batch * a.groups + 3) / 4;
  hipLaunchKernelGGL(k_group_norm_stats, dim3((unsigned)std::min<int64_t>(items, 4096)), dim3(256), 0, st, a, d.chunk);
  e = hipGetLastError();
  if (e != hipSuccess || a.rows <= 0) return e;
  hipLaunchKernelGGL((k_group_norm_rows<T, V>), dim3(d.chunks), dim3(d.threads), 0, st, a, d.chunk);
  return hipGetLastError();
}

template <typename T, int V, bool X8>
hipError_t backward(const GroupNormArgs& a, hipStream_t st) {
  const Deal d = deal(sizeof(T) == 2, a.rows, a.cols);
  hipLaunchKernelGGL((k_group_norm_bwd_sums<T, V, X8>), dim3(d.chunks), dim3(d.threads), sum_lds(d, a.cols, 2 * a.cols),
                     st, a, d.chunk);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int per = a.cols / a.groups, slice = std::max(1, BWD_COLS / per);
  const int blocks = (int)std::min<int64_t>((int64_t)a.batch * ((a.groups + slice - 1) / slice), 1 << 16);
  const int width = std::min(slice, a.groups) * per, lds = std::max(1024, std::max(1, 1024 / width) * width) * 4;
  hipLaunchKernelGGL(k_group_norm_bwd_means, dim3((unsigned)(blocks + 2 * ((a.cols + 63) / 64))), dim3(1024), lds, st, a,
                     d.chunk, d.chunks, blocks, slice);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_group_norm_bwd_rows<T, V, X8>), dim3(d.chunks), dim3(d.threads), 0, st, a, d.chunk);
  return hipGetLastError();
}

}  // namespace

size_t group_norm_workspace(bool bf16, int64_t rows, int32_t cols, int32_t groups, int32_t batch, bool backward) {
  if (rows <= 0) return 0;
  const Deal d = deal(bf16, rows, cols);
  const size_t pieces = (size_t)d.most + (size_t)batch;
  if (!backward) return pieces * 2 * (size_t)groups * 4;
  return ((pieces + (size_t)d.most) * 2 * (size_t)cols + 2 * (size_t)batch * (size_t)groups) * 4;
}

hipError_t launch_group_norm(bool bf16, const GroupNormArgs& a, hipStream_t st) {
  if (bf16) return a.cols < 8 ? forward<__bf16, 1>(a, st) : forward<__bf16, 8>(a, st);
  return a.cols < 4 ? forward<float, 1>(a, st) : forward<float, 4>(a, st);
}

hipError_t launch_group_norm_bwd(bool bf16, const GroupNormArgs& a, hipStream_t st) {
  if (a.rows <= 0 || a.batch <= 0) {  // sums over nothing
    const hipError_t e = a.dgain ? launch_fill_zero(a.dgain, (int64_t)a.cols * 4, st) : hipSuccess;
    return e == hipSuccess && a.dshift ? launch_fill_zero(a.dshift, (int64_t)a.cols * 4, st) : e;
  }
  const bool x8 = a.codes;
  if (bf16) {
    if (a.cols < 8) return x8 ? backward<__bf16, 1, true>(a, st) : backward<__bf16, 1, false>(a, st);
    return x8 ? backward<__bf16, 8, true>(a, st) : backward<__bf16, 8, false>(a, st);
  }
  if (a.cols < 4) return x8 ? backward<float, 1, true>(a, st) : backward<float, 1, false>(a, st);
  return x8 ? backward<float, 4, true>(a, st) : backward<float, 4, false>(a, st);
}

}  // namespace sscn
