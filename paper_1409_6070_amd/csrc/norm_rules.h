// How group norm's kernels deal rows: what device code and launch code share.  constexpr or plain,
// so a host program can run the same text.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <type_traits>

namespace sscn {

// Elements of a thread's vector: 16 bytes of x; in the backward pass 8 bytes of bf16, whose
// values and parameters take twice the registers (200001 rows of 100 in bf16 take 1.3 times as
// long with eight elements; forward, 589824 rows of 256 take 1.4 times as long with four).
inline int norm_vec(bool bf16, int cols, bool backward) {
  const int ve = bf16 && !backward ? 8 : 4;
  return cols < ve ? 1 : ve;
}

// Large samples: equal chunks of rows, one a workgroup.
struct NormDeal {
  int threads, rpb;
  int64_t chunk;
  int chunks, most;  // and a bound on them that grows with the rows
  bool join;         // few pieces a sample: they are joined by the last launch
};

// Workgroups, and rows of one, at least.  131072 x 512 backward from 8 bits: 43 + 68 us with 1024
// workgroups, with 512 56 + 77, with 2048 47 + 81; 60001 x 100 bf16 forward: 13 + 14 with 8 rows a
// thread, with 4 16.6 + 15.9, with 16 16.0 + 16.6.
inline NormDeal norm_deal(bool bf16, int64_t rows, int32_t cols, int32_t batch, bool backward) {
  const int v = norm_vec(bf16, cols, backward), nvec = (cols + v - 1) / v;
  NormDeal d;
  d.threads = nvec <= 256 ? 256 : v == 8 ? 512 : 1024;
  d.rpb = d.threads / nvec;
  const int64_t most = 1024 * 256 / d.threads;  // workgroups that the compute units hold at once
  const int64_t least = 8 * d.rpb;              // rows that pay for a workgroup's sums
  d.chunk = std::max(least, (rows + most - 1) / most);
  d.chunks = (int)((rows + d.chunk - 1) / d.chunk);
  d.most = (int)std::min(most, (rows + least - 1) / least);
  d.join = d.chunks <= 16 * (int64_t)batch;
  return d;
}

// A thread of nt among rows of nvec vectors: vector t of row lane rl of rpb.  Threads that are left
// over (on is false: nt may not be a multiple of nvec) have no row lane.
struct RowLane {
  int rl, rpb, t;
  bool on;
  constexpr inline RowLane(int thread, int nvec, int nt)
      : rl(thread / nvec), rpb(nt / nvec), t(thread - thread / nvec * nvec), on(thread / nvec < nt / nvec) {}
};

// The rows of a run of `count` that a thread takes: n of them, `all` that every thread has and
// `most` that any has.  A row lane without any stays at the run's last row.  Threads without a row lane
// load too, up to row all - 1 of theirs, and count from row 0: a further lane's would end one row
// behind the run where it is a multiple of rpb.
struct Share {
  int rl, n, all, most;
  constexpr inline Share(int count, int rl_, int rpb, bool on)
      : rl(!on ? 0 : rl_ < count - 1 ? rl_ : count - 1),
        n(on ? count / rpb + (rl_ < count - count / rpb * rpb ? 1 : 0) : 0),
        all(count / rpb),
        most(count / rpb + (count / rpb * rpb < count ? 1 : 0)) {}
};

// U of a thread's rows in flight.  take(q, k, valid) gets row k; `valid` is the constant true
// where every thread has that many.
template <class Q, int U>
struct Stream {
  Q q[U];
  template <class F>
  constexpr inline void fetch(const F& from, int i, int last) {
#pragma unroll
    for (int u = 0; u < U; ++u) from.load(q[u], i + u < last ? i + u : last);
  }
  // the first rows have been fetched
  template <class F, class Take>
  constexpr inline void run(const F& from, const Share& s, Take&& take) {
    int i = 0;
    for (; i + U <= s.all; i += U) {
#pragma unroll
      for (int u = 0; u < U; ++u) take(q[u], i + u, std::true_type{});
      if (i + 2 * U <= s.all) {
#pragma unroll
        for (int u = 0; u < U; ++u) from.load(q[u], i + U + u);
      } else if (i + U < s.most) {
        fetch(from, i + U, s.n > 1 ? s.n - 1 : 0);
      }
    }
    if (i < s.most)
#pragma unroll
      for (int u = 0; u < U; ++u) take(q[u], i + u, i + u < s.n);
  }
};

// Threads that share a column of `width` where a sample's pieces are joined, and the floats of LDS
// that they fill: two sums of every column from each.
constexpr inline int join_lanes(int nt, int width) { return nt / width > 1 ? nt / width : 1; }
constexpr inline int join_floats(int nt, int width) { return 2 * join_lanes(nt, width) * width; }

// The backward pass's means by a launch of their own, 1024 threads a workgroup: `slice` groups of a
// sample at a time (64 columns, but enough workgroups first), `blocks` workgroups, and their LDS: as
// much as any width up to the slice's fills, since the last slice may be narrower and its columns
// have more threads (2 groups of 9 fill 2016 floats, 3 only 1998).
struct NormMeans {
  int slice, blocks, floats;
};
inline NormMeans norm_means(int32_t batch, int32_t groups, int per) {
  NormMeans m;
  m.slice = (int)std::max<int64_t>(1, std::min<int64_t>(64 / per, (int64_t)batch * groups / 512));
  m.blocks = (int)std::min<int64_t>((int64_t)batch * ((groups + m.slice - 1) / m.slice), 1 << 16);
  m.floats = 2 * std::max(1024, std::min(m.slice, groups) * per);
  return m;
}

}  // namespace sscn
