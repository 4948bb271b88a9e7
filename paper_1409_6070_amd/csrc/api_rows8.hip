// C interface of group norm, rows held in 8 bits and their products.  Host code only:
// argument checks, workspace layout, launches on the caller's stream.

#include <cmath>

#include "sscn.h"
#include "common.h"
#include "kernels.h"
#include "checks.h"
#include "rows8.h"

using namespace sscn;

namespace {

// Rows that begin where a cache line does: kernels that write a row in several steps store
// past the caches only then (200001 rows of 300: a product's bf16 52 us, past them 67; 8-bit
// rows to float32 65 and 75).
bool whole_lines(const void* p, int64_t stride_bytes) { return (uintptr_t)p % 128 == 0 && stride_bytes % 128 == 0; }

bool cols8_ok(int32_t cols) { return cols >= 1 && cols <= SSCN_ROWS8_MAX_COLS; }

bool rows8_ok(const sscn_rows8* r) {
  return r && r->rows >= 0 && r->rows <= SSCN_MAX_ROWS && cols8_ok(r->cols) &&
         (r->rows == 0 || (r->d_codes && r->d_scales)) && (uintptr_t)r->d_codes % 16 == 0 &&
         (uintptr_t)r->d_scales % 4 == 0;
}

// The two arrays of 8-bit rows.
int64_t spans_of(const sscn_rows8& r, Span* list, bool out) {
  if (r.rows == 0) return 0;
  list[0] = span(r.d_codes, 1, r.rows * row8_code_stride(r.cols), 0, out);
  list[1] = span(r.d_scales, 1, r.rows * row8_scale_stride(r.cols), 0, out);
  return 2;
}

bool product_side_ok(int32_t n) { return n >= 1 && n <= SSCN_PRODUCT8_MAX; }

bool shape_ok(int32_t dtype, int64_t rows, int32_t cols, int32_t groups, int32_t batch) {
  return known_dtype(dtype) && rows >= 0 && rows <= SSCN_MAX_ROWS && cols >= 1 && cols <= SSCN_GROUP_NORM_MAX_COLS &&
         groups >= 1 && cols % groups == 0 && batch >= 0 &&
         batch <= SSCN_GROUP_NORM_MAX_BATCH;  // (sample numbers pass it by a grid's step in 32 bits)
}

sscn_status check_norm(const sscn_group_norm* n, bool backward) {
  if (!n || !shape_ok(n->dtype, n->rows, n->cols, n->groups, n->batch) || n->act < SSCN_ACT_NONE ||
      n->act > SSCN_ACT_SILU || !std::isfinite(n->eps) || !(n->eps > 0.f))
    return SSCN_ERR_INVALID_ARGUMENT;
  if (!n->d_begin && n->rows > 0 && (n->batch == 0 || n->rows % n->batch != 0)) return SSCN_ERR_INVALID_ARGUMENT;
  if (n->batch > 0 && !n->d_stats) return SSCN_ERR_INVALID_ARGUMENT;
  if (n->rows == 0) return SSCN_OK;
  if (n->d_x) return rows_ok(n->rows, n->cols, n->x_stride) ? SSCN_OK : SSCN_ERR_INVALID_ARGUMENT;
  const sscn_rows8 x{n->rows, n->cols, (uint8_t*)n->d_codes, (uint8_t*)n->d_scales};
  return backward && rows8_ok(&x) ? SSCN_OK : SSCN_ERR_INVALID_ARGUMENT;
}

// What forward and backward read besides dy, and the statistics.
int64_t norm_spans(const sscn_group_norm& n, Span* list, bool backward, int32_t in_place) {
  int64_t k = 0;
  const int64_t e = n.dtype == SSCN_BF16 ? 2 : 4;
  if (n.rows > 0 && n.d_x) list[k++] = span(n.d_x, n.rows, n.cols * e, n.x_stride * e, false, in_place);
  if (n.rows > 0 && !n.d_x)
    k += spans_of(sscn_rows8{n.rows, n.cols, (uint8_t*)n.d_codes, (uint8_t*)n.d_scales}, list + k, false);
  if (n.d_begin) list[k++] = span(n.d_begin, 1, ((int64_t)n.batch + 1) * 4, 0, false);
  if (n.d_gain) list[k++] = span(n.d_gain, 1, n.cols * 4, 0, false);
  if (n.d_shift) list[k++] = span(n.d_shift, 1, n.cols * 4, 0, false);
  if (n.batch > 0) list[k++] = span(n.d_stats, 1, (int64_t)n.batch * n.groups * 8, 0, !backward);
  return k;
}

GroupNormArgs args_of(const sscn_group_norm& n, void* ws) {
  GroupNormArgs a{};
  a.x = n.d_x;
  a.x_stride = n.x_stride;
  a.codes = n.d_x ? nullptr : n.d_codes;
  a.scales = n.d_x ? nullptr : n.d_scales;
  a.rows = n.rows;
  a.cols = n.cols;
  a.groups = n.groups;
  a.batch = n.batch;
  a.per = n.cols / n.groups;
  a.begin = n.d_begin;
  a.span = n.batch > 0 ? n.rows / n.batch : 0;
  a.gain = n.d_gain;
  a.shift = n.d_shift;
  a.eps = n.eps;
  a.slope = n.act == SSCN_ACT_NONE ? 1.f : n.act == SSCN_ACT_RELU ? 0.f : 1.f / 3.f;
  a.silu = n.act == SSCN_ACT_SILU;
  a.stream = n.rows * n.cols * (n.dtype == SSCN_BF16 ? 2 : 4) >= STREAM_BYTES;
  a.stats = n.d_stats;
  a.ws = (float*)ws;
  return a;
}

sscn_status product(int32_t dtype, const sscn_rows8* x, const void* d_weight8, size_t weight8_bytes, int32_t k,
                    int32_t n, bool transposed, const float* d_bias, void* d_y, int64_t y_stride, void* stream) {
  // (k: the sum's length, n: the result's columns)
  if (!known_dtype(dtype) || !rows8_ok(x) || !product_side_ok(k) || !product_side_ok(n) ||
      !rows_ok(x->rows, n, y_stride))
    return SSCN_ERR_INVALID_ARGUMENT;
  size_t need = 0;
  sscn_weight8_bytes(transposed ? n : k, transposed ? k : n, &need);
  if (bad_workspace(d_weight8, weight8_bytes, need)) return SSCN_ERR_WORKSPACE;
  if (x->rows == 0) return SSCN_OK;
  if (!d_y) return SSCN_ERR_INVALID_ARGUMENT;
  const int64_t e = dtype == SSCN_BF16 ? 2 : 4;
  const sscn_status overlap = apart(5, [&](Span* list) {
    int64_t c = spans_of(*x, list, false);
    list[c++] = span(d_weight8, 1, (int64_t)need, 0, false);
    if (d_bias) list[c++] = span(d_bias, 1, n * 4, 0, false);
    list[c++] = span(d_y, x->rows, n * e, y_stride * e, true);
    return c;
  });
  if (overlap != SSCN_OK) return overlap;
  const Weight8 w = weight8_parts((uint8_t*)d_weight8, transposed ? n : k, transposed ? k : n);
  Product8Args a{};
  a.x = x->d_codes;
  a.xs = x->d_scales;
  a.x_stride = row8_code_stride(k);
  a.xs_stride = row8_scale_stride(k);
  a.rows = x->rows;
  a.w = transposed ? w.codes : w.codes_t;
  a.ws = transposed ? w.scales : w.scales_t;
  a.w_stride = transposed ? w.stride : w.stride_t;
  a.ws_stride = transposed ? w.scale_stride : w.scale_stride_t;
  a.n = n;
  a.kb = (int32_t)row8_blocks(k);
  a.bias = d_bias;
  a.y = d_y;
  a.y_stride = y_stride;
  a.stream = a.rows * n * e >= STREAM_BYTES && whole_lines(d_y, y_stride * e);
  return of_hip(launch_product8(dtype == SSCN_BF16, a, (hipStream_t)stream));
}

}  // namespace

extern "C" {

sscn_status sscn_group_norm_workspace_bytes(int32_t dtype, int64_t rows, int32_t cols, int32_t groups, int32_t batch,
                                            int32_t backward, size_t* bytes) {
  if (!bytes || !shape_ok(dtype, rows, cols, groups, batch)) return SSCN_ERR_INVALID_ARGUMENT;
  *bytes = group_norm_workspace(dtype == SSCN_BF16, rows, cols, groups, batch, backward != 0);
  return SSCN_OK;
}

sscn_status sscn_group_norm_forward(const sscn_group_norm* norm, void* d_y, int64_t y_stride, void* d_workspace,
                                    size_t workspace_bytes, void* stream) {
  const sscn_status s = check_norm(norm, false);
  if (s != SSCN_OK) return s;
  const sscn_group_norm& n = *norm;
  if (!rows_ok(n.rows, n.cols, y_stride) || (n.rows > 0 && !d_y)) return SSCN_ERR_INVALID_ARGUMENT;
  const bool bf16 = n.dtype == SSCN_BF16;
  const size_t need = group_norm_workspace(bf16, n.rows, n.cols, n.groups, n.batch, false);
  if (bad_workspace(d_workspace, workspace_bytes, need)) return SSCN_ERR_WORKSPACE;
  const sscn_status overlap = apart(8, [&](Span* list) {
    int64_t k = norm_spans(n, list, false, 0);
    const int64_t e = bf16 ? 2 : 4;
    if (n.rows > 0) list[k++] = span(d_y, n.rows, n.cols * e, y_stride * e, true, 0);
    if (need) list[k++] = span(d_workspace, 1, (int64_t)need, 0, true);
    return k;
  });
  if (overlap != SSCN_OK) return overlap;
  GroupNormArgs a = args_of(n, d_workspace);
  a.y = d_y;
  a.y_stride = y_stride;
  return of_hip(launch_group_norm(bf16, a, (hipStream_t)stream));
}

sscn_status sscn_group_norm_backward(const sscn_group_norm* norm, const void* d_dy, int64_t dy_stride, void* d_dx,
                                     int64_t dx_stride, float* d_dgain, float* d_dshift, void* d_workspace,
                                     size_t workspace_bytes, void* stream) {
  const sscn_status s = check_norm(norm, true);
  if (s != SSCN_OK) return s;
  const sscn_group_norm& n = *norm;
  if (!rows_ok(n.rows, n.cols, dy_stride) || !rows_ok(n.rows, n.cols, dx_stride) || (n.rows > 0 && (!d_dy || !d_dx)))
    return SSCN_ERR_INVALID_ARGUMENT;
  const bool bf16 = n.dtype == SSCN_BF16;
  const size_t need = group_norm_workspace(bf16, n.rows, n.cols, n.groups, n.batch, true);
  if (bad_workspace(d_workspace, workspace_bytes, need)) return SSCN_ERR_WORKSPACE;
  const sscn_status overlap = apart(11, [&](Span* list) {
    int64_t k = norm_spans(n, list, true, 0);
    const int64_t e = bf16 ? 2 : 4;
    if (n.rows > 0) {
      list[k++] = span(d_dy, n.rows, n.cols * e, dy_stride * e, false, 0);
      list[k++] = span(d_dx, n.rows, n.cols * e, dx_stride * e, true, 0);
    }
    if (d_dgain) list[k++] = span(d_dgain, 1, n.cols * 4, 0, true);
    if (d_dshift) list[k++] = span(d_dshift, 1, n.cols * 4, 0, true);
    if (need) list[k++] = span(d_workspace, 1, (int64_t)need, 0, true);
    return k;
  });
  if (overlap != SSCN_OK) return overlap;
  GroupNormArgs a = args_of(n, d_workspace);
  a.dy = d_dy;
  a.dy_stride = dy_stride;
  a.dx = d_dx;
  a.dx_stride = dx_stride;
  a.dgain = d_dgain;
  a.dshift = d_dshift;
  return of_hip(launch_group_norm_bwd(bf16, a, (hipStream_t)stream));
}

sscn_status sscn_rows8_strides(int32_t cols, int64_t* code_stride, int64_t* scale_stride) {
  if (!cols8_ok(cols) || !code_stride || !scale_stride) return SSCN_ERR_INVALID_ARGUMENT;
  *code_stride = row8_code_stride(cols);
  *scale_stride = row8_scale_stride(cols);
  return SSCN_OK;
}

sscn_status sscn_rows8_store(int32_t dtype, const void* d_x, int64_t x_stride, const sscn_rows8* to, void* stream) {
  if (!known_dtype(dtype) || !rows8_ok(to) || !rows_ok(to->rows, to->cols, x_stride)) return SSCN_ERR_INVALID_ARGUMENT;
  if (to->rows == 0) return SSCN_OK;
  if (!d_x) return SSCN_ERR_INVALID_ARGUMENT;
  const int64_t e = dtype == SSCN_BF16 ? 2 : 4;
  const sscn_status overlap = apart(3, [&](Span* list) {
    list[0] = span(d_x, to->rows, to->cols * e, x_stride * e, false);
    return 1 + spans_of(*to, list + 1, true);
  });
  if (overlap != SSCN_OK) return overlap;
  Rows8Args a{};
  a.x = d_x;
  a.x_stride = x_stride;
  a.rows = to->rows;
  a.cols = to->cols;
  a.codes = to->d_codes;
  a.scales = to->d_scales;
  return of_hip(launch_rows8_store(dtype == SSCN_BF16, a, (hipStream_t)stream));
}

sscn_status sscn_rows8_load(int32_t dtype, const sscn_rows8* from, void* d_y, int64_t y_stride, void* stream) {
  if (!known_dtype(dtype) || !rows8_ok(from) || !rows_ok(from->rows, from->cols, y_stride))
    return SSCN_ERR_INVALID_ARGUMENT;
  if (from->rows == 0) return SSCN_OK;
  if (!d_y) return SSCN_ERR_INVALID_ARGUMENT;
  const int64_t e = dtype == SSCN_BF16 ? 2 : 4;
  const sscn_status overlap = apart(3, [&](Span* list) {
    list[0] = span(d_y, from->rows, from->cols * e, y_stride * e, true);
    return 1 + spans_of(*from, list + 1, false);
  });
  if (overlap != SSCN_OK) return overlap;
  Rows8Args a{};
  a.rows = from->rows;
  a.cols = from->cols;
  a.codes = from->d_codes;
  a.scales = from->d_scales;
  a.y = d_y;
  a.y_stride = y_stride;
  a.stream = a.rows * a.cols * e >= STREAM_BYTES && (e == 2 || whole_lines(d_y, y_stride * e));
  return of_hip(launch_rows8_load(dtype == SSCN_BF16, a, (hipStream_t)stream));
}

sscn_status sscn_weight8_bytes(int32_t k, int32_t n, size_t* bytes) {
  if (!product_side_ok(k) || !product_side_ok(n) || !bytes) return SSCN_ERR_INVALID_ARGUMENT;
  int64_t b = 0;
  weight8_parts(nullptr, k, n, &b);
  *bytes = (size_t)b;
  return SSCN_OK;
}

sscn_status sscn_weight8_store(int32_t dtype, const void* d_w, int64_t w_stride, int32_t k, int32_t n, void* d_weight8,
                               size_t weight8_bytes, void* stream) {
  size_t need = 0;
  if (!known_dtype(dtype) || !d_w || sscn_weight8_bytes(k, n, &need) != SSCN_OK || !rows_ok(k, n, w_stride))
    return SSCN_ERR_INVALID_ARGUMENT;
  if (bad_workspace(d_weight8, weight8_bytes, need)) return SSCN_ERR_WORKSPACE;
  const int64_t e = dtype == SSCN_BF16 ? 2 : 4;
  const sscn_status overlap = apart(2, [&](Span* list) {
    list[0] = span(d_w, k, n * e, w_stride * e, false);
    list[1] = span(d_weight8, 1, (int64_t)need, 0, true);
    return (int64_t)2;
  });
  if (overlap != SSCN_OK) return overlap;
  Weight8Args a{};
  a.w = d_w;
  a.w_stride = w_stride;
  a.k = k;
  a.n = n;
  a.w8 = (uint8_t*)d_weight8;
  return of_hip(launch_weight8_store(dtype == SSCN_BF16, a, (hipStream_t)stream));
}

sscn_status sscn_product8_forward(int32_t dtype, const sscn_rows8* x, const void* d_weight8, size_t weight8_bytes,
                                  int32_t n, const float* d_bias, void* d_y, int64_t y_stride, void* stream) {
  if (!x) return SSCN_ERR_INVALID_ARGUMENT;
  return product(dtype, x, d_weight8, weight8_bytes, x->cols, n, false, d_bias, d_y, y_stride, stream);
}

sscn_status sscn_product8_input_grad(int32_t dtype, const sscn_rows8* dy, const void* d_weight8, size_t weight8_bytes,
                                     int32_t k, void* d_dx, int64_t dx_stride, void* stream) {
  if (!dy) return SSCN_ERR_INVALID_ARGUMENT;
  return product(dtype, dy, d_weight8, weight8_bytes, dy->cols, k, true, nullptr, d_dx, dx_stride, stream);
}

sscn_status sscn_product8_weight_grad_workspace_bytes(int64_t rows, int32_t k, int32_t n, size_t* bytes) {
  if (rows < 0 || rows > SSCN_MAX_ROWS || !product_side_ok(k) || !product_side_ok(n) || !bytes)
    return SSCN_ERR_INVALID_ARGUMENT;
  const size_t splits = (size_t)weight_grad8_most_splits(rows, k, n);
  *bytes = splits > 1 ? splits * ((size_t)k + 1) * (size_t)n * 4 : 0;
  return SSCN_OK;
}

sscn_status sscn_product8_weight_grad(const sscn_rows8* x, const sscn_rows8* dy, float* d_dw, int64_t dw_stride,
                                      float* d_db, void* d_workspace, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  if (!rows8_ok(x) || !rows8_ok(dy) || x->rows != dy->rows || !d_dw ||
      sscn_product8_weight_grad_workspace_bytes(x->rows, x->cols, dy->cols, &need) != SSCN_OK ||
      !rows_ok(x->cols, dy->cols, dw_stride))
    return SSCN_ERR_INVALID_ARGUMENT;
  if (bad_workspace(d_workspace, workspace_bytes, need)) return SSCN_ERR_WORKSPACE;
  const sscn_status overlap = apart(7, [&](Span* list) {
    int64_t c = spans_of(*x, list, false);
    c += spans_of(*dy, list + c, false);
    list[c++] = span(d_dw, x->cols, (int64_t)dy->cols * 4, dw_stride * 4, true);
    if (d_db) list[c++] = span(d_db, 1, (int64_t)dy->cols * 4, 0, true);
    if (need) list[c++] = span(d_workspace, 1, (int64_t)need, 0, true);
    return c;
  });
  if (overlap != SSCN_OK) return overlap;
  WeightGrad8Args a{};
  a.x = x->d_codes;
  a.xs = x->d_scales;
  a.x_stride = row8_code_stride(x->cols);
  a.xs_stride = row8_scale_stride(x->cols);
  a.dy = dy->d_codes;
  a.dys = dy->d_scales;
  a.dy_stride = row8_code_stride(dy->cols);
  a.dys_stride = row8_scale_stride(dy->cols);
  a.rows = x->rows;
  a.k = x->cols;
  a.n = dy->cols;
  a.dw = d_dw;
  a.dw_stride = dw_stride;
  a.db = d_db;
  a.part = need ? (float*)d_workspace : nullptr;
  return of_hip(launch_weight_grad8(a, (hipStream_t)stream));
}

}  // extern "C"
