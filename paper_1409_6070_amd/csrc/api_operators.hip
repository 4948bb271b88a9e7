// C interface of the operators that need no network: layer norm, orthogonalised
// matrices and the update that uses them.  Host code only: argument checks,
// workspace layout, launches on the caller's stream.

#include <algorithm>
#include <cmath>
#include <cstring>
#include <memory>
#include <new>

#include "sscn.h"
#include "common.h"
#include "kernels.h"
#include "spans.h"

using namespace sscn;

namespace {

bool known_dtype(int32_t dtype) { return dtype == SSCN_F32 || dtype == SSCN_BF16; }

size_t aligned256(size_t n) { return (n + 255) / 256 * 256; }

sscn_status of_hip(hipError_t e) { return e == hipSuccess ? SSCN_OK : SSCN_ERR_HIP; }

// Elements from an array's first to its last, at most: their bytes fit 63 bits.
constexpr int64_t MAX_SPAN = (int64_t)1 << 60;

// rows x cols elements with `stride` elements between rows (both below 2^32: no overflow here)
bool rows_ok(int64_t rows, int64_t cols, int64_t stride) {
  return rows >= 0 && rows <= SSCN_MAX_ROWS && stride >= cols && stride <= ((int64_t)1 << 31) &&
         (rows <= 1 || (rows - 1) * stride + cols <= MAX_SPAN);
}

bool norm_ok(int32_t dtype, int64_t rows, int32_t cols, float eps) {
  return known_dtype(dtype) && rows >= 0 && rows <= SSCN_MAX_ROWS && cols >= 1 && cols <= SSCN_NORM_MAX_COLS &&
         std::isfinite(eps) && eps > 0.f;
}

bool shape_ok(int64_t rows, int64_t cols) {
  return rows >= 1 && cols >= 1 && std::min(rows, cols) <= SSCN_ORTHO_MAX_SHORT && std::max(rows, cols) <= SSCN_ORTHO_MAX_LONG;
}

// The exponent of two that brings values up to `most` within NS_PLANE.
int32_t plane_exponent(double most) {
  return most > 0.0 ? (int32_t)std::min(60.0, std::floor(std::log2(NS_PLANE / most))) : 0;
}

// Follows the singular values that start in [0, 1] through the steps.  Each step's
// largest |p(s)| and |b s^2 + c s^4| over [0, hi] lie at hi or where the derivative is
// zero; entries of X, A and B are at most hi, hi^2 and the latter.  Sets out[0 .. steps - 1]
// and returns true if X stays within 3.5 and B within 200.
bool follow_steps(int32_t steps, const float* coef, NsStep (&out)[SSCN_ORTHO_MAX_STEPS]) {
  if (steps < 1 || steps > SSCN_ORTHO_MAX_STEPS || !coef) return false;
  double hi = 1.0;
  for (int k = 0; k < steps; ++k) {
    const double a = coef[3 * k], b = coef[3 * k + 1], c = coef[3 * k + 2];
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
    double most = 0.0, inner = 0.0;
    const double end = hi * hi;
    auto at = [&](double q) {  // q = s^2
      if (!(q >= 0.0 && q <= end)) return;
      const double p = b * q + c * q * q;
      inner = std::max(inner, std::fabs(p));
      most = std::max(most, std::fabs(a + p) * std::sqrt(q));
    };
    at(end);
    if (c != 0.0) at(-b / (2.0 * c));
    // a + 3 b q + 5 c q^2 = 0, its roots without a difference of nearly equal numbers:
    // where c is too small to matter the cubic's extremum is still one of them
    const double d = 9.0 * b * b - 20.0 * a * c;
    if (d >= 0.0) {
      const double t = -0.5 * (3.0 * b + std::copysign(std::sqrt(d), b));
      if (c != 0.0) at(t / (5.0 * c));
      if (t != 0.0) at(a / t);
    }
    if (!(inner <= 200.0) || !(most <= 3.5)) return false;
    out[k] = NsStep{coef[3 * k], coef[3 * k + 1], coef[3 * k + 2], plane_exponent(hi), plane_exponent(end),
                    plane_exponent(inner)};
    hi = most;
  }
  return true;
}

// Workspace of one matrix; sets its pointers when base is not null.
size_t carve_matrix(NsMat& M, int64_t rows, int64_t cols, char* base) {
  M.tall = rows > cols;
  M.m = (int32_t)std::min(rows, cols);
  M.n = (int32_t)std::max(rows, cols);
  M.mp = (int32_t)round_up(M.m, 32);
  M.np = (int32_t)round_up(M.n, 32);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* p = base ? base + off : nullptr;
    off += aligned256(bytes);
    return p;
  };
  const size_t x = (size_t)M.mp * M.np * 4, g = (size_t)M.mp * M.mp * 4;
  M.X = (float*)take(x);
  M.opX = take(x);
  M.opXt[0] = take(x);
  M.opXt[1] = take(x);
  M.opA = take(g);
  M.opB = take(g);
  M.ssq = (double*)take(NS_SSQ * sizeof(double));
  return off;
}

// Matrices go through the launches in groups of NS_MATS, which share the workspace.
// Carves a group's part of it, the matrices with the longest sums first, and calls
// fill(index, matrix) for each; returns the bytes.
template <class Shape, class Fill>
size_t carve_group(NsGroup& g, int32_t first, int k, Shape&& shape, Fill&& fill, char* base) {
  size_t off = 0;
  g.a.n = k;
  for (int j = 0; j < k; ++j) {
    NsMat& M = g.t.mat[j];
    M = NsMat{};
    const auto s = shape(first + j);
    off += carve_matrix(M, s.first, s.second, base ? base + off : nullptr);
    fill(first + j, M);
  }
  std::stable_sort(g.t.mat, g.t.mat + k, [](const NsMat& x, const NsMat& y) { return x.n > y.n; });
  g.a.table = (const NsTable*)(base ? base + off : nullptr);
  off += aligned256(sizeof(NsTable));
  g.a.count = (int32_t*)(base ? base + off : nullptr);
  off += aligned256(NS_COUNT * sizeof(int32_t));
  g.a.part = (float*)(base ? base + off : nullptr);
  return off + aligned256(ns_part_bytes(g));
}

template <class Shape>
size_t group_bytes(int32_t n, Shape&& shape) {
  size_t most = 0;
  NsGroup g{};
  for (int32_t i = 0; i < n; i += NS_MATS)
    most = std::max(most, carve_group(g, i, std::min(NS_MATS, n - i), shape, [](int32_t, NsMat&) {}, nullptr));
  return most;
}

template <class Shape, class Fill>
hipError_t run_groups(int32_t n, Shape&& shape, Fill&& fill, NsGroup& g, bool bf16, bool muon, int32_t steps,
                      const NsStep* step, void* d_ws, hipStream_t st) {
  for (int32_t i = 0; i < n; i += NS_MATS) {
    carve_group(g, i, std::min(NS_MATS, n - i), shape, fill, (char*)d_ws);
    const hipError_t e = launch_newton_schulz(g, bf16, muon, steps, step, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

bool bad_workspace(const void* ws, size_t have, size_t need) {
  return need > 0 && (!ws || have < need || (uintptr_t)ws % 256 != 0);
}

// Refuses arrays of which one that is written overlaps another: fill(list) sets at most
// `most` of them and returns how many.
template <class Fill>
sscn_status apart(int64_t most, Fill&& fill) {
  Span few[64];
  std::unique_ptr<Span[]> many;
  Span* list = few;
  if (most > 64) {
    many.reset(new (std::nothrow) Span[most]);
    if (!many) return SSCN_ERR_INVALID_ARGUMENT;
    list = many.get();
  }
  return outputs_overlap(list, fill(list)) ? SSCN_ERR_INVALID_ARGUMENT : SSCN_OK;
}

}  // namespace

extern "C" {

sscn_status sscn_layer_norm_forward(int32_t dtype, const void* d_x, int64_t x_stride, int64_t rows, int32_t cols,
                                    const float* d_gain, const float* d_shift, float eps, void* d_y, int64_t y_stride,
                                    void* stream) {
  if (!norm_ok(dtype, rows, cols, eps) || !rows_ok(rows, cols, x_stride) || !rows_ok(rows, cols, y_stride))
    return SSCN_ERR_INVALID_ARGUMENT;
  if (rows == 0) return SSCN_OK;
  if (!d_x || !d_y) return SSCN_ERR_INVALID_ARGUMENT;
  const int64_t e = dtype == SSCN_BF16 ? 2 : 4;
  const sscn_status overlap = apart(4, [&](Span* list) {
    int64_t k = 0;
    list[k++] = span(d_x, rows, cols * e, x_stride * e, false, 0);
    list[k++] = span(d_y, rows, cols * e, y_stride * e, true, 0);
    if (d_gain) list[k++] = span(d_gain, 1, cols * 4, 0, false);
    if (d_shift) list[k++] = span(d_shift, 1, cols * 4, 0, false);
    return k;
  });
  if (overlap != SSCN_OK) return overlap;
  NormArgs a{};
  a.x = d_x;
  a.x_stride = x_stride;
  a.rows = rows;
  a.cols = cols;
  a.gain = d_gain;
  a.shift = d_shift;
  a.eps = eps;
  a.y = d_y;
  a.y_stride = y_stride;
  a.y_cols = cols;
  return of_hip(launch_norm(dtype == SSCN_BF16, a, (hipStream_t)stream));
}

sscn_status sscn_layer_norm_workspace_bytes(int32_t dtype, int64_t rows, int32_t cols, size_t* bytes) {
  if (!bytes || !norm_ok(dtype, rows, cols, 1.f)) return SSCN_ERR_INVALID_ARGUMENT;
  *bytes = (size_t)norm_parts(dtype == SSCN_BF16, rows, cols) * (size_t)cols * 2 * sizeof(float);
  return SSCN_OK;
}

sscn_status sscn_layer_norm_backward(int32_t dtype, const void* d_dy, int64_t dy_stride, const void* d_x,
                                     int64_t x_stride, int64_t rows, int32_t cols, const float* d_gain, float eps,
                                     void* d_dx, int64_t dx_stride, float* d_dgain, float* d_dshift, void* d_workspace,
                                     size_t workspace_bytes, void* stream) {
  if (!norm_ok(dtype, rows, cols, eps) || !rows_ok(rows, cols, dy_stride) || !rows_ok(rows, cols, x_stride) ||
      !rows_ok(rows, cols, dx_stride))
    return SSCN_ERR_INVALID_ARGUMENT;
  if (rows > 0 && (!d_dy || !d_x || !d_dx)) return SSCN_ERR_INVALID_ARGUMENT;
  const bool params = d_dgain || d_dshift;
  size_t need = 0;
  if (params && rows > 0) sscn_layer_norm_workspace_bytes(dtype, rows, cols, &need);
  if (bad_workspace(d_workspace, workspace_bytes, need)) return SSCN_ERR_WORKSPACE;
  const int64_t e = dtype == SSCN_BF16 ? 2 : 4;
  const sscn_status overlap = apart(7, [&](Span* list) {
    int64_t k = 0;
    if (rows > 0) {
      list[k++] = span(d_dy, rows, cols * e, dy_stride * e, false, 0);
      list[k++] = span(d_x, rows, cols * e, x_stride * e, false, 0);
      list[k++] = span(d_dx, rows, cols * e, dx_stride * e, true, 0);
    }
    if (d_gain) list[k++] = span(d_gain, 1, cols * 4, 0, false);
    if (d_dgain) list[k++] = span(d_dgain, 1, cols * 4, 0, true);
    if (d_dshift) list[k++] = span(d_dshift, 1, cols * 4, 0, true);
    if (need) list[k++] = span(d_workspace, 1, (int64_t)need, 0, true);
    return k;
  });
  if (overlap != SSCN_OK) return overlap;
  NormBwdArgs a{};
  a.dy = d_dy;
  a.dy_stride = dy_stride;
  a.x = d_x;
  a.x_stride = x_stride;
  a.rows = rows;
  a.cols = cols;
  a.gain = d_gain;
  a.eps = eps;
  a.dx = d_dx;
  a.dx_stride = dx_stride;
  a.dx_cols = cols;
  a.part = need ? (float*)d_workspace : nullptr;
  return of_hip(launch_norm_bwd(dtype == SSCN_BF16, false, a, d_dgain, d_dshift, (hipStream_t)stream));
}

sscn_status sscn_orthogonalize_workspace_bytes(int32_t n, const sscn_ortho_matrix* h_matrices, size_t* bytes) {
  if (n < 0 || (n > 0 && !h_matrices) || !bytes) return SSCN_ERR_INVALID_ARGUMENT;
  for (int32_t i = 0; i < n; ++i)
    if (!shape_ok(h_matrices[i].rows, h_matrices[i].cols)) return SSCN_ERR_INVALID_ARGUMENT;
  *bytes = group_bytes(n, [&](int32_t i) { return std::make_pair(h_matrices[i].rows, h_matrices[i].cols); });
  return SSCN_OK;
}

sscn_status sscn_orthogonalize(int32_t dtype, int32_t n, const sscn_ortho_matrix* h_matrices, int32_t steps,
                               const float* h_coef, void* d_workspace, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  NsStep step[SSCN_ORTHO_MAX_STEPS];
  if (!known_dtype(dtype) || !follow_steps(steps, h_coef, step)) return SSCN_ERR_INVALID_ARGUMENT;
  const sscn_status s = sscn_orthogonalize_workspace_bytes(n, h_matrices, &need);
  if (s != SSCN_OK) return s;
  for (int32_t i = 0; i < n; ++i) {
    const sscn_ortho_matrix& m = h_matrices[i];
    if (!m.d_in || !m.d_out || !rows_ok(m.rows, m.cols, m.in_stride) || !rows_ok(m.rows, m.cols, m.out_stride))
      return SSCN_ERR_INVALID_ARGUMENT;
  }
  if (bad_workspace(d_workspace, workspace_bytes, need)) return SSCN_ERR_WORKSPACE;
  const sscn_status overlap = apart((int64_t)n * 2 + 1, [&](Span* list) {
    const int64_t e = dtype == SSCN_BF16 ? 2 : 4;
    int64_t k = 0;
    for (int32_t i = 0; i < n; ++i) {
      const sscn_ortho_matrix& m = h_matrices[i];
      list[k++] = span(m.d_in, m.rows, m.cols * e, m.in_stride * e, false, i);
      list[k++] = span(m.d_out, m.rows, m.cols * e, m.out_stride * e, true, i);
    }
    if (need) list[k++] = span(d_workspace, 1, (int64_t)need, 0, true);
    return k;
  });
  if (overlap != SSCN_OK) return overlap;
  NsGroup g{};
  return of_hip(run_groups(
      n, [&](int32_t i) { return std::make_pair(h_matrices[i].rows, h_matrices[i].cols); },
      [&](int32_t i, NsMat& M) {
        M.u = h_matrices[i].d_in;
        M.u_stride = h_matrices[i].in_stride;
        M.o = h_matrices[i].d_out;
        M.o_stride = h_matrices[i].out_stride;
      },
      g, dtype == SSCN_BF16, false, steps, step, d_workspace, (hipStream_t)stream));
}

sscn_status sscn_muon_workspace_bytes(int32_t n, const sscn_muon_param* h_params, size_t* bytes) {
  if (n < 0 || (n > 0 && !h_params) || !bytes) return SSCN_ERR_INVALID_ARGUMENT;
  // in the groups of sscn_muon_update: NS_MATS orthogonalised matrices at a time, in order
  size_t most = 0;
  for (int32_t i = 0; i < n;) {
    int64_t shape[NS_MATS][2];
    int k = 0;
    for (; i < n && k < NS_MATS; ++i) {
      const sscn_muon_param& p = h_params[i];
      if (p.orthogonal) {
        if (!shape_ok(p.rows, p.cols)) return SSCN_ERR_INVALID_ARGUMENT;
        shape[k][0] = p.rows;
        shape[k++][1] = p.cols;
      } else if (p.rows < 1 || p.cols < 1 || p.rows > SSCN_MAX_ROWS || p.cols > SSCN_MAX_ROWS ||
                 p.rows * p.cols > MAX_SPAN) {
        return SSCN_ERR_INVALID_ARGUMENT;
      }
    }
    most = std::max(most, group_bytes(k, [&](int32_t j) { return std::make_pair(shape[j][0], shape[j][1]); }));
  }
  *bytes = most;
  return SSCN_OK;
}

sscn_status sscn_muon_update(int32_t dtype, int32_t n, const sscn_muon_param* h_params, float momentum, int32_t nesterov,
                             int32_t steps, const float* h_coef, void* d_workspace, size_t workspace_bytes,
                             void* stream) {
  if (!known_dtype(dtype) || !(momentum >= 0.f) || !std::isfinite(momentum)) return SSCN_ERR_INVALID_ARGUMENT;
  size_t need = 0;
  const sscn_status s = sscn_muon_workspace_bytes(n, h_params, &need);
  if (s != SSCN_OK) return s;
  bool any = false;
  for (int32_t i = 0; i < n; ++i) {
    const sscn_muon_param& p = h_params[i];
    if (!p.d_w || !p.d_g || !p.d_v || !(p.lr >= 0.f) || !std::isfinite(p.lr) || !(p.weight_decay >= 0.f) ||
        !std::isfinite(p.weight_decay) || !std::isfinite(p.scale))
      return SSCN_ERR_INVALID_ARGUMENT;
    any = any || p.orthogonal;
  }
  NsStep step[SSCN_ORTHO_MAX_STEPS];
  if (any && !follow_steps(steps, h_coef, step)) return SSCN_ERR_INVALID_ARGUMENT;
  if (bad_workspace(d_workspace, workspace_bytes, need)) return SSCN_ERR_WORKSPACE;
  const sscn_status overlap = apart((int64_t)n * 4 + 1, [&](Span* list) {
    int64_t k = 0;
    for (int32_t i = 0; i < n; ++i) {
      const sscn_muon_param& p = h_params[i];
      const int64_t bytes = p.rows * p.cols * 4;
      list[k++] = span(p.d_w, 1, bytes, 0, true);
      list[k++] = span(p.d_v, 1, bytes, 0, true);
      list[k++] = span(p.d_g, 1, bytes, 0, false);
      if (p.d_w_store && p.d_w_store != (void*)p.d_w)
        list[k++] = span(p.d_w_store, 1, dtype == SSCN_BF16 ? bytes / 2 : bytes, 0, true);
    }
    if (need) list[k++] = span(d_workspace, 1, (int64_t)need, 0, true);
    return k;
  });
  if (overlap != SSCN_OK) return overlap;
  hipStream_t st = (hipStream_t)stream;
  SgdArgs sgd;
  std::memset((void*)&sgd, 0, sizeof(sgd));
  sgd.store_bf16 = dtype == SSCN_BF16;
  sgd.momentum = momentum;
  auto flush = [&]() {
    const hipError_t e = launch_sgd(sgd, st);
    sgd.njobs = 0;
    sgd.blk_beg[0] = 0;
    return e;
  };
  NsGroup g{};
  g.a.momentum = momentum;
  g.a.nesterov = nesterov != 0;
  const sscn_muon_param* group[NS_MATS];
  int k = 0;
  auto flush_group = [&]() {
    const hipError_t e = run_groups(
        k, [&](int32_t j) { return std::make_pair(group[j]->rows, group[j]->cols); },
        [&](int32_t j, NsMat& M) {
          const sscn_muon_param& p = *group[j];
          M.u = p.d_g;
          M.w = p.d_w;
          M.v = p.d_v;
          M.o = p.d_w_store == (void*)p.d_w ? nullptr : p.d_w_store;
          M.scale = p.lr * p.scale;
          M.decay = p.lr * p.weight_decay;
        },
        g, dtype == SSCN_BF16, true, steps, step, d_workspace, st);
    k = 0;
    return e;
  };
  for (int32_t i = 0; i < n; ++i) {
    const sscn_muon_param& p = h_params[i];
    if (p.orthogonal) {
      group[k++] = &p;
      if (k == NS_MATS && flush_group() != hipSuccess) return SSCN_ERR_HIP;
      continue;
    }
    SgdJob& J = sgd.job[sgd.njobs];
    J.w = p.d_w;
    J.w_store = p.d_w_store == (void*)p.d_w ? nullptr : p.d_w_store;
    J.g = p.d_g;
    J.v = p.d_v;
    J.n = p.rows * p.cols;
    J.wd = p.weight_decay;
    J.lr = p.lr;
    const int blocks = (int)std::max<int64_t>(1, std::min<int64_t>(2048, (J.n + 255) / 256));
    sgd.blk_beg[sgd.njobs + 1] = sgd.blk_beg[sgd.njobs] + blocks;
    if (++sgd.njobs == MAX_SGD_JOBS && flush() != hipSuccess) return SSCN_ERR_HIP;
  }
  if (sgd.njobs && flush() != hipSuccess) return SSCN_ERR_HIP;
  return of_hip(k ? flush_group() : hipSuccess);
}

}  // extern "C"
