// Host side of the operators around a language model's residual stream and its sampling: argument checks and the order of their launches.
// Nothing is enqueued when an argument is refused.
#include <cmath>

#include "dw_ops_checks.h"

using namespace dw;

namespace {

inline bool shape_ok(int64_t rows, int64_t n) { return rows >= 0 && rows < kMaxRows && n >= 1 && n <= DW_MAX_NORM; }
// the table gradient's (2^24 blocks of 256 threads are too many for a launch)
inline bool grad_rows_ok(int64_t rows, int64_t n) { return rows <= 1 << 27 && rows * n <= 1ll << 36; }
inline bool share_ok(float p) { return p >= 0.f && p <= 1.f; }

// a 16-bit number below the limit keeps an element
Drop drop_of(float p, uint64_t seed, uint64_t step, const uint64_t* d_step) {
  Drop d;
  d.limit = (uint32_t)std::lround((1.0 - (double)p) * 65536.0);
  d.factor = d.limit ? (float)(65536.0 / (double)d.limit) : 0.f;
  d.seed = seed;
  d.step = step;
  d.d_step = d.limit < 65536u ? d_step : nullptr;
  return d;
}

// an output that may be an input's own rows
inline bool same_rows_or_other(const void* out, int64_t out_ld, int64_t out_stride, const void* in, int64_t ld, int64_t stride, int k, int64_t rows) {
  return out != in || ((rows <= 1 || out_ld == ld) && (k == 1 || out_stride == stride));
}

}  // namespace

extern "C" {

int dw_embedding(const int32_t* d_token, const void* d_table, int64_t table_ld, int64_t table_stride, int table_dtype, int k,
                 int64_t rows, int64_t vocab, int64_t n, int dtype, float scale, void* d_y, int64_t y_ld, int64_t y_stride,
                 void* stream) {
  if (k < 1 || k > DW_MAX_K || !is_type(dtype) || !is_type(table_dtype)) return DW_ERR_CONFIG;
  if (!shape_ok(rows, n) || vocab < 1 || vocab > DW_MAX_VOCAB) return DW_ERR_ARG;
  if (!std::isfinite(scale)) return DW_ERR_HYPER;
  if (rows == 0) return DW_OK;
  if (!d_token || !d_table || !d_y) return DW_ERR_NULL;
  if (!aligned(d_token, 4) || !in_ok(d_table, table_ld, table_stride, vocab, n, type_bytes(table_dtype))) return DW_ERR_ARG;
  if (d_y == d_table || !out_ok(d_y, y_ld, y_stride, k, rows, n, type_bytes(dtype))) return DW_ERR_ARG;
  EmbedArgs a = {};
  a.token = d_token;
  a.table = {d_table, table_ld, table_stride};
  a.y = {d_y, y_ld, y_stride};
  a.k = k; a.rows = rows; a.vocab = vocab; a.n = n; a.scale = scale;
  DW_HIP(launch_embedding(a, table_dtype, dtype, (hipStream_t)stream));
  return DW_OK;
}

size_t dw_embedding_grad_scratch_bytes(int k, int64_t rows, int64_t vocab, int64_t n) {
  if (k < 1 || k > DW_MAX_K || !shape_ok(rows, n) || vocab < 1 || vocab > DW_MAX_VOCAB || rows == 0 || !grad_rows_ok(rows, n)) return 0;
  return embedding_grad_scratch(k, rows, vocab, n);
}

int dw_embedding_grad(const void* d_dy, int64_t dy_ld, int64_t dy_stride, const int32_t* d_token, int k, int64_t rows,
                      int64_t vocab, int64_t n, int dtype, float scale, int accumulate, float* d_grad, int64_t grad_ld,
                      int64_t grad_stride, void* d_scratch, size_t scratch_bytes, void* stream) {
  if (k < 1 || k > DW_MAX_K || !is_type(dtype)) return DW_ERR_CONFIG;
  if (!shape_ok(rows, n) || vocab < 1 || vocab > DW_MAX_VOCAB || (accumulate != 0 && accumulate != 1)) return DW_ERR_ARG;
  if (!std::isfinite(scale)) return DW_ERR_HYPER;
  if (!grad_rows_ok(rows, n)) return DW_ERR_TOO_LARGE;
  if (rows == 0 && accumulate) return DW_OK;
  if (!d_grad) return DW_ERR_NULL;
  if (!out_ok(d_grad, grad_ld, grad_stride, k, vocab, n, 4)) return DW_ERR_ARG;
  if (rows > 0) {
    if (!d_dy || !d_token) return DW_ERR_NULL;
    if (!aligned(d_token, 4) || d_dy == d_grad || !in_ok(d_dy, dy_ld, dy_stride, rows, n, type_bytes(dtype))) return DW_ERR_ARG;
    if (!d_scratch || !aligned(d_scratch, 256) || scratch_bytes < dw_embedding_grad_scratch_bytes(k, rows, vocab, n)) return DW_ERR_WORKSPACE;
  }
  EmbedGradArgs a = {};
  a.token = d_token;
  a.dy = {d_dy, dy_ld, dy_stride};
  a.grad = d_grad; a.grad_ld = vocab == 1 ? n : grad_ld; a.grad_stride = grad_stride;
  a.k = k; a.accumulate = accumulate; a.rows = rows; a.vocab = vocab; a.n = n; a.scale = scale;
  a.scratch = static_cast<char*>(d_scratch);
  DW_HIP(launch_embedding_grad(a, dtype, (hipStream_t)stream));
  return DW_OK;
}

int dw_dropout(const void* d_x, int64_t x_ld, int64_t x_stride, const void* d_residual, int64_t residual_ld,
               int64_t residual_stride, int k, int64_t rows, int64_t n, int dtype, float p, uint64_t seed, uint64_t step,
               const uint64_t* d_step, void* d_y, int64_t y_ld, int64_t y_stride, void* stream) {
  if (k < 1 || k > DW_MAX_K || !is_type(dtype)) return DW_ERR_CONFIG;
  if (!shape_ok(rows, n)) return DW_ERR_ARG;
  if (!share_ok(p)) return DW_ERR_HYPER;
  if (rows == 0) return DW_OK;
  if (!d_x || !d_y) return DW_ERR_NULL;
  const int64_t b = type_bytes(dtype);
  if (!in_ok(d_x, x_ld, x_stride, rows, n, b) || !out_ok(d_y, y_ld, y_stride, k, rows, n, b) || !aligned(d_step, 8)) return DW_ERR_ARG;
  if (d_residual && !in_ok(d_residual, residual_ld, residual_stride, rows, n, b)) return DW_ERR_ARG;
  if (!same_rows_or_other(d_y, y_ld, y_stride, d_x, x_ld, x_stride, k, rows) ||
      !same_rows_or_other(d_y, y_ld, y_stride, d_residual, residual_ld, residual_stride, k, rows)) return DW_ERR_ARG;
  DropoutArgs a = {};
  a.x = {d_x, x_ld, x_stride};
  a.res = {d_residual, residual_ld, residual_stride};
  a.y = {d_y, y_ld, y_stride};
  a.drop = drop_of(p, seed, step, d_step);
  a.k = k; a.rows = rows; a.n = n;
  DW_HIP(launch_dropout(a, dtype, (hipStream_t)stream));
  return DW_OK;
}

int dw_rms_norm(const void* d_x, int64_t x_ld, int64_t x_stride, const void* d_residual, int64_t residual_ld,
                int64_t residual_stride, const float* d_gamma, int64_t param_stride, int k, int64_t rows, int64_t n, int dtype,
                float eps, float p, uint64_t seed, uint64_t step, const uint64_t* d_step, void* d_h, int64_t h_ld,
                int64_t h_stride, void* d_y, int64_t y_ld, int64_t y_stride, uint8_t* d_q, uint8_t* d_scale, uint8_t* d_qt,
                uint8_t* d_scale_t, float* d_rstd, void* stream) {
  if (k < 1 || k > DW_MAX_K || !is_type(dtype)) return DW_ERR_CONFIG;
  if (!shape_ok(rows, n) || ((d_q || d_qt) && rows > DW_MAX_FP8)) return DW_ERR_ARG;
  if (!(eps >= 0.f) || !std::isfinite(eps) || !share_ok(p)) return DW_ERR_HYPER;
  if (rows == 0) return DW_OK;
  const Drop drop = drop_of(p, seed, step, d_step);
  const bool changed = d_residual || drop.limit < 65536u;   // h is not x
  if (!d_x || (!d_y && !d_q && !d_qt && !d_h && !d_rstd) || (d_q && !d_scale) || (d_qt && (!d_scale_t || !d_rstd || (changed && !d_h))))
    return DW_ERR_NULL;
  const int64_t b = type_bytes(dtype);
  if (!in_ok(d_x, x_ld, x_stride, rows, n, b) || !params_ok(d_gamma, param_stride) || !aligned(d_step, 8) || !aligned(d_rstd, 4)) return DW_ERR_ARG;
  if (d_residual && !in_ok(d_residual, residual_ld, residual_stride, rows, n, b)) return DW_ERR_ARG;
  if (d_h && (!out_ok(d_h, h_ld, h_stride, k, rows, n, b) || !same_rows_or_other(d_h, h_ld, h_stride, d_x, x_ld, x_stride, k, rows) ||
              !same_rows_or_other(d_h, h_ld, h_stride, d_residual, residual_ld, residual_stride, k, rows))) return DW_ERR_ARG;
  if (d_y && (d_y == d_x || d_y == d_residual || d_y == d_h || !out_ok(d_y, y_ld, y_stride, k, rows, n, b))) return DW_ERR_ARG;
  if (!aligned(d_q, 16) || !aligned(d_qt, 16) || !aligned(d_scale, 4) || !aligned(d_scale_t, 4)) return DW_ERR_ARG;
  RmsArgs a = {};
  a.x = {d_x, x_ld, x_stride};
  a.res = {d_residual, residual_ld, residual_stride};
  a.drop = drop;
  a.gamma = d_gamma; a.param_stride = param_stride;
  a.h = {d_h, h_ld, h_stride};
  a.y = {d_y, y_ld, y_stride};
  a.q = d_q; a.scale = d_scale;
  a.rstd = d_rstd;
  a.k = k; a.rows = rows; a.n = n; a.eps = eps;
  DW_HIP(launch_rms_norm(a, dtype, (hipStream_t)stream));
  if (!d_qt) return DW_OK;
  QuantArgs t = {};
  t.x = d_h ? Rows{d_h, h_ld, h_stride} : Rows{d_x, x_ld, x_stride};
  t.k = k; t.rows = rows; t.n = n;
  t.qt = d_qt; t.scale_t = d_scale_t;
  t.rstd = d_rstd;
  t.gamma = d_gamma; t.gamma_stride = param_stride;
  DW_HIP(launch_fp8_quantize(t, dtype, (hipStream_t)stream));
  return DW_OK;
}

size_t dw_rms_norm_grad_scratch_bytes(int k, int64_t rows, int64_t n, int dtype) {
  if (k < 1 || k > DW_MAX_K || !is_type(dtype) || !shape_ok(rows, n)) return 0;
  return (size_t)k * rms_norm_grad_strips(k, rows, n, dtype) * n * sizeof(float);
}

int dw_rms_norm_grad(const void* d_dy, int64_t dy_ld, int64_t dy_stride, const void* d_h, int64_t h_ld, int64_t h_stride,
                     const float* d_gamma, int64_t param_stride, const float* d_rstd, const void* d_dh, int64_t dh_ld,
                     int64_t dh_stride, int k, int64_t rows, int64_t n, int dtype, float p, uint64_t seed, uint64_t step,
                     const uint64_t* d_step, void* d_dres, int64_t dres_ld, int64_t dres_stride, void* d_dx, int64_t dx_ld,
                     int64_t dx_stride, float* d_dgamma, int64_t grad_stride, void* d_scratch, size_t scratch_bytes,
                     void* stream) {
  if (k < 1 || k > DW_MAX_K || !is_type(dtype)) return DW_ERR_CONFIG;
  if (!shape_ok(rows, n)) return DW_ERR_ARG;
  if (!share_ok(p)) return DW_ERR_HYPER;
  if (!d_dres && !d_dx && !d_dgamma) return DW_OK;
  if (d_dgamma && !grads_ok(d_dgamma, grad_stride, k, n)) return DW_ERR_ARG;
  if (rows == 0 && !d_dgamma) return DW_OK;
  const int64_t b = type_bytes(dtype);
  if (rows > 0) {
    if (!d_dy || !d_h || !d_rstd) return DW_ERR_NULL;
    if (!in_ok(d_dy, dy_ld, dy_stride, rows, n, b) || !in_ok(d_h, h_ld, h_stride, rows, n, b) ||
        (d_dh && !in_ok(d_dh, dh_ld, dh_stride, rows, n, b))) return DW_ERR_ARG;
    if (!params_ok(d_gamma, param_stride) || !aligned(d_rstd, 4) || !aligned(d_step, 8)) return DW_ERR_ARG;
    if (d_dres && (d_dres == d_h || d_dres == d_dx || !out_ok(d_dres, dres_ld, dres_stride, k, rows, n, b) ||
                   !same_rows_or_other(d_dres, dres_ld, dres_stride, d_dy, dy_ld, dy_stride, k, rows) ||
                   !same_rows_or_other(d_dres, dres_ld, dres_stride, d_dh, dh_ld, dh_stride, k, rows))) return DW_ERR_ARG;
    if (d_dx && (d_dx == d_h || d_dx == d_dh || !out_ok(d_dx, dx_ld, dx_stride, k, rows, n, b) ||
                 !same_rows_or_other(d_dx, dx_ld, dx_stride, d_dy, dy_ld, dy_stride, k, rows))) return DW_ERR_ARG;
    if (d_dgamma && (!d_scratch || !aligned(d_scratch, 256) || scratch_bytes < dw_rms_norm_grad_scratch_bytes(k, rows, n, dtype)))
      return DW_ERR_WORKSPACE;
  }
  RmsGradArgs a = {};
  a.dy = {d_dy, dy_ld, dy_stride};
  a.h = {d_h, h_ld, h_stride};
  a.dh = {d_dh, dh_ld, dh_stride};
  a.drop = drop_of(p, seed, step, d_step);
  a.gamma = d_gamma; a.param_stride = param_stride;
  a.rstd = d_rstd;
  a.dres = {d_dres, dres_ld, dres_stride};
  a.dx = {d_dx, dx_ld, dx_stride};
  a.dgamma = d_dgamma; a.grad_stride = grad_stride;
  a.part = d_dgamma ? static_cast<float*>(d_scratch) : nullptr;
  a.k = k; a.rows = rows; a.n = n;
  a.strips = rms_norm_grad_strips(k, rows, n, dtype);
  DW_HIP(launch_rms_norm_grad(a, dtype, (hipStream_t)stream));
  return DW_OK;
}

int dw_adjust_logits(const void* d_logits, int64_t ld, int64_t stride, const int32_t* d_history, int64_t history_ld,
                     int64_t history_stride, int64_t length, const int32_t* d_filled, const int32_t* d_answer,
                     const float* d_repetition, const float* d_presence, const float* d_frequency, const float* d_bias,
                     int64_t bias_ld, int64_t bias_stride, const uint32_t* d_mask, int64_t mask_ld, int64_t mask_stride, int k,
                     int64_t rows, int64_t vocab, int dtype, void* d_out, int64_t out_ld, int64_t out_stride, void* stream) {
  if (k < 1 || k > DW_MAX_K || !is_type(dtype)) return DW_ERR_CONFIG;
  if (rows < 0 || rows >= kMaxRows || vocab < 1 || vocab > DW_MAX_VOCAB || length < 0 || length > DW_MAX_HISTORY) return DW_ERR_ARG;
  if (rows == 0) return DW_OK;
  if (!d_logits || !d_out || (length > 0 && !d_history)) return DW_ERR_NULL;
  const int64_t b = type_bytes(dtype);
  if (!in_ok(d_logits, ld, stride, rows, vocab, b) || !out_ok(d_out, out_ld, out_stride, k, rows, vocab, b) ||
      !same_rows_or_other(d_out, out_ld, out_stride, d_logits, ld, stride, k, rows)) return DW_ERR_ARG;
  if (!aligned(d_filled, 4) || !aligned(d_answer, 4) || !aligned(d_repetition, 4) || !aligned(d_presence, 4) || !aligned(d_frequency, 4)) return DW_ERR_ARG;
  // rows that are only read may be one for all
  if (length > 0 && !in_ok(d_history, history_ld, history_stride, history_ld == 0 ? 1 : rows, length, 4)) return DW_ERR_ARG;
  if (d_bias && !in_ok(d_bias, bias_ld, bias_stride, bias_ld == 0 ? 1 : rows, vocab, 4)) return DW_ERR_ARG;
  if (d_mask && !in_ok(d_mask, mask_ld, mask_stride, mask_ld == 0 ? 1 : rows, ceil_div(vocab, 32), 4)) return DW_ERR_ARG;
  AdjustArgs a = {};
  a.logits = {d_logits, ld, stride};
  a.out = {d_out, out_ld, out_stride};
  a.history = length > 0 ? d_history : nullptr; a.history_ld = history_ld; a.history_stride = history_stride; a.length = length;
  a.filled = d_filled; a.answer = d_answer;
  a.repetition = d_repetition; a.presence = d_presence; a.frequency = d_frequency;
  a.bias = d_bias; a.bias_ld = bias_ld; a.bias_stride = bias_stride;
  a.mask = d_mask; a.mask_ld = mask_ld; a.mask_stride = mask_stride;
  a.k = k; a.rows = rows; a.vocab = vocab;
  DW_HIP(launch_adjust_logits(a, dtype, (hipStream_t)stream));
  return DW_OK;
}

}  // extern "C"
