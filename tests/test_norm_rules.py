"""How group norm's kernels deal rows and LDS, compiled for the host: the addresses that they read, which no result
shows (no GPU)."""
from tests.test_host_rules import run_host

ROWS = r"""
#include "norm_rules.h"
#include <cstdio>
#include <vector>
using namespace sscn;
// A thread's rows of a run that starts at row lo: `least` and `most` of those that it loads.
struct Row { int64_t row; };
struct Rows {
  int64_t first; int step;
  int64_t* least; int64_t* most;
  void load(Row& q, int k) const {
    q.row = first + (int64_t)k * step;
    if (q.row < *least) *least = q.row;
    if (q.row > *most) *most = q.row;
  }
};
static std::vector<unsigned char> taken;
// A workgroup of nt threads, rows of nvec vectors, over rows 0 .. whole - 1 of which 0 .. count - 1 are its
// first piece: the first rows are fetched before the piece is known, as the kernels do.
template <int U> bool piece(int nt, int nvec, int whole, int count, int rows, bool row_by_row) {
  taken.assign(count, 0);
  const int lanes = (nt + nvec - 1) / nvec;
  for (int l = 0; l < lanes; ++l)  // (the vectors of a row lane read the same rows)
    for (int last = 0; last < 2; ++last) {
      const int thread = last ? std::min(nt, (l + 1) * nvec) - 1 : l * nvec;
      const RowLane p(thread, nvec, nt);
      if (p.rpb != nt / nvec || p.on != (p.rl < p.rpb) || p.t < 0 || p.t >= nvec || p.rl * nvec + p.t != thread) return false;
      const Share w(whole, p.rl, p.rpb, p.on), h(count, p.rl, p.rpb, p.on);
      int64_t least = 0, most = 0;
      Stream<Row, U> s;
      s.fetch(Rows{w.rl, p.rpb, &least, &most}, 0, w.n > 1 ? w.n - 1 : 0);
      if (least < 0 || most >= rows) return false;  // (rows of the array)
      least = most = 0;
      if (row_by_row) s.fetch(Rows{h.rl, p.rpb, &least, &most}, 0, h.n > 1 ? h.n - 1 : 0);
      bool good = true;
      s.run(Rows{h.rl, p.rpb, &least, &most}, h, [&](const Row& q, int k, auto valid) {
        if (!p.on || !valid) return;
        const int64_t row = h.rl + (int64_t)k * p.rpb;
        good = good && q.row == row && row < count && k < h.n;
        if (good && !last) good = taken[row]++ == 0;
      });
      if (!good || least < 0 || most >= count) return false;  // rows of the piece
    }
  for (int r = 0; r < count; ++r)
    if (!taken[r]) return false;
  return true;
}
template <int U> long pieces(int nt, int nvec, int chunk) {
  const int rpb = nt / nvec;
  long n = 0;
  std::vector<int> counts = {1, 2, rpb - 1, rpb, rpb + 1, chunk - 1, chunk, chunk + 1};
  for (int k = 1; k <= 4; ++k)
    for (int d = -1; d <= 1; ++d)
      for (int off : {d, d * rpb}) counts.push_back(k * U * rpb + off);
  for (int count : counts) {
    if (count < 1) continue;
    for (int whole : {count, count + 1, count + rpb}) {
      if (!piece<U>(nt, nvec, whole, count, whole, whole != count && n % 2)) {
        printf("%d threads, %d vectors, %d of %d rows, %d in flight\n", nt, nvec, count, whole, U);
        return -1;
      }
      ++n;
    }
  }
  return n;
}
int main() {
  long n = 0;
  bool seen[1025][2049] = {};
  for (int cols = 1; cols <= 4096; ++cols)
    for (int form = 0; form < 4; ++form) {
      const int v = norm_vec(form & 1, cols, form & 2), nvec = (cols + v - 1) / v;
      const NormDeal d = norm_deal(form & 1, 100000, cols, 100, form & 2);
      if (seen[d.threads][nvec]) continue;
      seen[d.threads][nvec] = true;
      for (int64_t chunk : {(int64_t)8 * d.rpb, d.chunk}) {
        const long a = pieces<8>(d.threads, nvec, (int)chunk), b = pieces<4>(d.threads, nvec, (int)chunk);
        if (a < 0 || b < 0) return 1;
        n += a + b;
      }
    }
  printf("%ld\n", n);
}
"""


def test_rows_stay_in_their_piece(tmp_path):
    """Every load of every thread, also of those that have no row or no vector of one, over rows of 1 to 4096
    columns and runs around multiples of the rows in flight; every row is taken once."""
    assert int(run_host(tmp_path, ROWS)) > 100000


MEANS = r"""
#include "norm_rules.h"
#include <cstdio>
using namespace sscn;
int main() {
  long n = 0;
  for (int per = 1; per <= 4096; ++per)
    for (int groups = 1; groups * per <= 4096; groups = groups < 70 ? groups + 1 : groups + groups / 9)
      for (int batch : {1, 2, 5, 8, 31, 60, 63, 100, 700, 5000}) {
        const NormMeans m = norm_means(batch, groups, per);
        if (m.slice < 1 || m.blocks < 1 || m.floats < 1024) return 1;  // (1024: the parameters' sums)
        for (int g0 = 0; g0 < groups; g0 += m.slice) {  // the last slice may be narrower
          const int width = std::min(m.slice, groups - g0) * per;
          if (2 * std::max(1, 1024 / width) * width > m.floats) {
            printf("%d groups of %d, batch %d: %d columns in %d floats\n", groups, per, batch, width, m.floats);
            return 1;
          }
        }
        ++n;
      }
  printf("%ld\n", n);
}
"""


def test_joined_means_stay_in_their_lds(tmp_path):
    """[2][lanes of a column][columns] floats of every slice of groups that a workgroup joins."""
    assert int(run_host(tmp_path, MEANS)) > 100000
