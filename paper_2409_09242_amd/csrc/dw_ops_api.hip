// Host side of the operators for training steps that the caller puts together: argument checks and the order of their launches.  Nothing is
// enqueued when an argument is refused.
#include <cmath>

#include "dw_ops.h"

using namespace dw;

namespace {

#define DW_HIP(expr)                                          \
  do {                                                        \
    hipError_t e__ = (expr);                                  \
    if (e__ != hipSuccess) return note_hip_error(e__);        \
  } while (0)

inline bool is_type(int dtype) { return dtype == DW_F32 || dtype == DW_BF16; }
inline int64_t type_bytes(int dtype) { return dtype == DW_BF16 ? 2 : 4; }
inline bool aligned(const void* p, int64_t a) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(a - 1)) == 0; }

constexpr int64_t kMaxRows = 1ll << 31;                     // rows of a worker
constexpr int64_t kMaxStride = 1ll << 48;                   // elements: a byte offset stays in 64 bits for every worker

// rows of n at p that are only read
inline bool in_ok(const void* p, int64_t ld, int64_t stride, int64_t rows, int64_t n, int64_t bytes) {
  return aligned(p, bytes) && (rows <= 1 || ld >= n) && ld >= 0 && ld <= kMaxStride / (rows > 0 ? rows : 1) && stride >= 0 && stride <= kMaxStride;
}
// no two rows of k workers share an element (a worker's own do not, ld >= n): the workers lie one behind the other, or each row
// of a worker between two of worker 0's, or behind its last one
inline bool rows_apart(int64_t ld, int64_t stride, int k, int64_t rows, int64_t n) {
  if (k == 1 || rows == 0 || stride >= (rows - 1) * ld + n) return true;
  for (int w = 1; w < k; ++w) {                             // (what holds for the first rows of two workers holds for all w apart)
    const int64_t at = w * stride;
    const int64_t before = rows == 1 || at >= (rows - 1) * ld ? rows - 1 : at / ld;        // the last row of worker 0 that begins at or before
    if (at - before * ld < n || (before + 1 < rows && (before + 1) * ld - at < n)) return false;
  }
  return true;
}
// rows that are written: no two of them share an element
inline bool out_ok(const void* p, int64_t ld, int64_t stride, int k, int64_t rows, int64_t n, int64_t bytes) {
  return in_ok(p, ld, stride, rows, n, bytes) && rows_apart(ld, stride, k, rows, n);
}
inline bool params_ok(const float* p, int64_t stride) { return aligned(p, 4) && stride >= 0 && stride <= kMaxStride; }
inline bool grads_ok(const float* p, int64_t stride, int k, int64_t n) { return params_ok(p, stride) && (k == 1 || stride >= n); }

inline bool norm_shape_ok(int k, int64_t rows, int64_t n) {
  return rows >= 0 && rows < kMaxRows && n >= 1 && n <= DW_MAX_NORM;
}

inline bool fp8_product_fits(int k, int64_t m, int64_t n) { return ceil_div(m, 64) * ceil_div(n, 64) * k <= (1 << 22); }   // one grid

struct ClipSizes { int64_t elements, chunk; int parts; };   // of one worker
int clip_sizes(int k, int n_tensors, const int64_t* h_count, ClipSizes* z) {
  if (k < 1 || k > DW_MAX_K) return DW_ERR_CONFIG;
  if (n_tensors < 0 || n_tensors > DW_MAX_TENSORS) return DW_ERR_ARG;
  if (!h_count && n_tensors > 0) return DW_ERR_NULL;
  z->elements = 0;
  for (int j = 0; j < n_tensors; ++j) {
    if (h_count[j] < 0 || h_count[j] > (1ll << 40)) return DW_ERR_ARG;
    z->elements += h_count[j];
  }
  if (z->elements > (1ll << 40)) return DW_ERR_ARG;
  z->chunk = clip_chunk(z->elements * k);
  int64_t parts = 0;
  for (int j = 0; j < n_tensors; ++j) parts += ceil_div(h_count[j], z->chunk);
  z->parts = (int)parts;                                    // at most 16384 + DW_MAX_TENSORS
  return DW_OK;
}

}  // namespace

extern "C" {

int dw_layer_norm(const void* d_x, int64_t x_ld, int64_t x_stride, const float* d_gamma, const float* d_beta,
                  int64_t param_stride, int k, int64_t rows, int64_t n, int dtype, float eps, void* d_y, int64_t y_ld,
                  int64_t y_stride, float* d_mean, float* d_rstd, void* stream) {
  if (k < 1 || k > DW_MAX_K || !is_type(dtype)) return DW_ERR_CONFIG;
  if (!norm_shape_ok(k, rows, n)) return DW_ERR_ARG;
  if (!(eps >= 0.f) || !std::isfinite(eps)) return DW_ERR_HYPER;
  if (rows == 0) return DW_OK;
  if (!d_x || !d_y) return DW_ERR_NULL;
  const int64_t b = type_bytes(dtype);
  if (d_y == d_x || !in_ok(d_x, x_ld, x_stride, rows, n, b) || !out_ok(d_y, y_ld, y_stride, k, rows, n, b)) return DW_ERR_ARG;
  if (!params_ok(d_gamma, param_stride) || !params_ok(d_beta, param_stride)) return DW_ERR_ARG;
  if (!aligned(d_mean, 4) || !aligned(d_rstd, 4)) return DW_ERR_ARG;
  NormArgs a = {};
  a.x = {d_x, x_ld, x_stride};
  a.out = {d_y, y_ld, y_stride};
  a.gamma = d_gamma; a.beta = d_beta; a.param_stride = param_stride;
  a.mean = d_mean; a.rstd = d_rstd;
  a.k = k; a.rows = rows; a.n = n; a.eps = eps;
  DW_HIP(launch_layer_norm(a, dtype, (hipStream_t)stream));
  return DW_OK;
}

size_t dw_layer_norm_grad_scratch_bytes(int k, int64_t rows, int64_t n, int dtype) {
  if (k < 1 || k > DW_MAX_K || !is_type(dtype) || !norm_shape_ok(k, rows, n)) return 0;
  return (size_t)k * layer_norm_grad_strips(k, rows, n, dtype) * 2 * n * sizeof(float);
}

int dw_layer_norm_grad(const void* d_dy, int64_t dy_ld, int64_t dy_stride, const void* d_x, int64_t x_ld, int64_t x_stride,
                       const float* d_gamma, int64_t param_stride, const float* d_mean, const float* d_rstd, int k,
                       int64_t rows, int64_t n, int dtype, void* d_dx, int64_t dx_ld, int64_t dx_stride, float* d_dgamma,
                       float* d_dbeta, int64_t grad_stride, void* d_scratch, size_t scratch_bytes, void* stream) {
  if (k < 1 || k > DW_MAX_K || !is_type(dtype)) return DW_ERR_CONFIG;
  if (!norm_shape_ok(k, rows, n)) return DW_ERR_ARG;
  const bool sums = d_dgamma || d_dbeta;
  if (!d_dx && !sums) return DW_OK;
  if (sums && (!grads_ok(d_dgamma, grad_stride, k, n) || !grads_ok(d_dbeta, grad_stride, k, n) || d_dgamma == d_dbeta)) return DW_ERR_ARG;
  if (rows == 0 && !sums) return DW_OK;
  const int64_t b = type_bytes(dtype);
  if (rows > 0) {
    if (!d_dy || !d_x || !d_mean || !d_rstd) return DW_ERR_NULL;
    if (!in_ok(d_dy, dy_ld, dy_stride, rows, n, b) || !in_ok(d_x, x_ld, x_stride, rows, n, b)) return DW_ERR_ARG;
    if (d_dx && (d_dx == d_dy || d_dx == d_x || !out_ok(d_dx, dx_ld, dx_stride, k, rows, n, b))) return DW_ERR_ARG;
    if (!params_ok(d_gamma, param_stride) || !aligned(d_mean, 4) || !aligned(d_rstd, 4)) return DW_ERR_ARG;
    if (sums && (!d_scratch || !aligned(d_scratch, 256) || scratch_bytes < dw_layer_norm_grad_scratch_bytes(k, rows, n, dtype)))
      return DW_ERR_WORKSPACE;
  }
  NormArgs a = {};
  a.x = {d_x, x_ld, x_stride};
  a.dy = {d_dy, dy_ld, dy_stride};
  a.out = {d_dx, dx_ld, dx_stride};
  a.gamma = d_gamma; a.param_stride = param_stride;
  a.mean = const_cast<float*>(d_mean); a.rstd = const_cast<float*>(d_rstd);
  a.dgamma = d_dgamma; a.dbeta = d_dbeta; a.grad_stride = grad_stride;
  a.part = sums ? static_cast<float*>(d_scratch) : nullptr;
  a.k = k; a.rows = rows; a.n = n;
  a.strips = layer_norm_grad_strips(k, rows, n, dtype);
  DW_HIP(launch_layer_norm_grad(a, sums, dtype, (hipStream_t)stream));
  return DW_OK;
}

int dw_token_logp(const void* d_logits, int64_t ld, int64_t stride, const int32_t* d_target, int k, int64_t rows,
                  int64_t vocab, int dtype, float* d_logp, void* stream) {
  if (k < 1 || k > DW_MAX_K || !is_type(dtype)) return DW_ERR_CONFIG;
  if (rows < 0 || rows >= kMaxRows || vocab < 1 || vocab > DW_MAX_VOCAB) return DW_ERR_ARG;
  if (rows == 0) return DW_OK;
  if (!d_logits || !d_target || !d_logp) return DW_ERR_NULL;
  if (!in_ok(d_logits, ld, stride, rows, vocab, type_bytes(dtype)) || !aligned(d_target, 4) || !aligned(d_logp, 4)) return DW_ERR_ARG;
  PolicyArgs a = {};
  a.logits = {d_logits, ld, stride};
  a.target = d_target;
  a.mean_weight = 1.f;
  a.logp = d_logp;
  a.k = k; a.rows = rows; a.vocab = vocab;
  DW_HIP(launch_policy(a, dtype, (hipStream_t)stream));
  return DW_OK;
}

size_t dw_policy_loss_scratch_bytes(int k, int64_t rows) {
  if (k < 1 || k > DW_MAX_K || rows < 0 || rows >= kMaxRows) return 0;
  return (size_t)k * rows * sizeof(float);
}

int dw_policy_loss(const void* d_logits, int64_t ld, int64_t stride, const int32_t* d_target, const float* d_old_logp,
                   const float* d_ref_logp, const float* d_advantage, const float* d_weight, int k, int64_t rows,
                   int64_t vocab, int dtype, float clip_low, float clip_high, float kl_coef, float* d_loss, float* d_logp,
                   void* d_grad, int64_t grad_ld, int64_t grad_stride, void* d_scratch, size_t scratch_bytes, void* stream) {
  if (k < 1 || k > DW_MAX_K || !is_type(dtype)) return DW_ERR_CONFIG;
  if (rows < 0 || rows >= kMaxRows || vocab < 1 || vocab > DW_MAX_VOCAB) return DW_ERR_ARG;
  if (!(clip_low >= 0.f && clip_low <= 1.f) || !(clip_high >= 0.f) || !std::isfinite(clip_high) || !std::isfinite(kl_coef)) return DW_ERR_HYPER;
  if (!aligned(d_loss, 4) || !aligned(d_logp, 4)) return DW_ERR_ARG;
  if (rows > 0) {
    if (!d_logits || !d_target || !d_old_logp || !d_advantage || (kl_coef != 0.f && !d_ref_logp)) return DW_ERR_NULL;
    const int64_t b = type_bytes(dtype);
    if (!in_ok(d_logits, ld, stride, rows, vocab, b) || !aligned(d_target, 4)) return DW_ERR_ARG;
    if (!aligned(d_old_logp, 4) || !aligned(d_ref_logp, 4) || !aligned(d_advantage, 4) || !aligned(d_weight, 4)) return DW_ERR_ARG;
    if (d_grad && !out_ok(d_grad, grad_ld, grad_stride, k, rows, vocab, b)) return DW_ERR_ARG;
    if (d_grad == d_logits && (grad_ld != ld || (k > 1 && grad_stride != stride))) return DW_ERR_ARG;      // in place: the same rows
    if (d_loss && (!d_scratch || !aligned(d_scratch, 256) || scratch_bytes < dw_policy_loss_scratch_bytes(k, rows))) return DW_ERR_WORKSPACE;
  }
  PolicyArgs a = {};
  a.logits = {d_logits, ld, stride};
  a.grad = {d_grad, grad_ld, grad_stride};
  a.target = d_target;
  a.old_logp = d_old_logp; a.ref_logp = d_ref_logp; a.advantage = d_advantage;
  a.weight = d_weight;
  a.mean_weight = rows > 0 ? 1.f / (float)rows : 0.f;
  a.q_min = 1.f - clip_low; a.q_max = 1.f + clip_high; a.kl_coef = kl_coef;
  a.logp = d_logp;
  a.part = d_loss ? static_cast<float*>(d_scratch) : nullptr;
  a.loss = d_loss;
  a.k = k; a.rows = rows; a.vocab = vocab;
  DW_HIP(launch_policy(a, dtype, (hipStream_t)stream));
  return DW_OK;
}

size_t dw_clip_grads_scratch_bytes(int k, int n_tensors, const int64_t* h_count) {
  ClipSizes z;
  if (clip_sizes(k, n_tensors, h_count, &z) != DW_OK) return 0;
  return (size_t)k * (z.parts + 1) * sizeof(double);       // the partial sums, and the norms
}

int dw_clip_grads(const void* const* h_grad, const int64_t* h_count, const int32_t* h_dtype, int k, int n_tensors, int dtype,
                  float max_norm, float* d_out, int64_t out_stride, float* d_norm, void* d_scratch, size_t scratch_bytes,
                  void* stream) {
  ClipSizes z;
  const int st = clip_sizes(k, n_tensors, h_count, &z);
  if (st != DW_OK) return st;
  if (!h_dtype && !is_type(dtype)) return DW_ERR_CONFIG;
  for (int j = 0; h_dtype && j < n_tensors; ++j)
    if (!is_type(h_dtype[j])) return DW_ERR_CONFIG;
  if (!(max_norm > 0.f)) return DW_ERR_HYPER;
  if (!d_norm || (!h_grad && z.elements > 0)) return DW_ERR_NULL;
  if (!aligned(d_norm, 4) || (d_out && !grads_ok(d_out, out_stride, k, z.elements))) return DW_ERR_ARG;
  for (int w = 0; w < k; ++w)
    for (int j = 0; j < n_tensors; ++j) {
      const void* g = h_grad ? h_grad[(int64_t)w * n_tensors + j] : nullptr;
      if (h_count[j] == 0) continue;
      if (!g) return DW_ERR_NULL;
      if (!aligned(g, type_bytes(h_dtype ? h_dtype[j] : dtype))) return DW_ERR_ARG;
    }
  if ((!d_scratch || !aligned(d_scratch, 256) || scratch_bytes < dw_clip_grads_scratch_bytes(k, n_tensors, h_count)))
    return DW_ERR_WORKSPACE;
  const hipStream_t s = (hipStream_t)stream;
  double* part = static_cast<double*>(d_scratch);
  const bool writes = z.parts > 0 && (d_out || std::isfinite(max_norm));
  double* wide = clip_adds_in_between(z.parts) ? part + (int64_t)k * z.parts : nullptr;
  // first pass over all tensors, then the second: both in launches of as many tensors as the arguments hold
  for (int pass = 0; pass < (writes ? 2 : 1); ++pass) {
    if (pass == 1 && wide) DW_HIP(launch_grad_norm(part, z.parts, d_norm, wide, k, s));
    ClipTable t;
    t.wide = wide;
    t.chunk = z.chunk;
    t.part = part; t.parts = z.parts; t.part0 = 0;
    t.norm = d_norm; t.max_norm = max_norm;
    t.out = d_out; t.out_stride = out_stride; t.out0 = 0;
    t.worker0 = 0; t.workers = k;
    const int most = ClipTable::tensors(k);
    for (int j0 = 0; j0 < n_tensors; j0 += most) {
      t.n = n_tensors - j0 < most ? n_tensors - j0 : most;
      clip_table_fill(t, h_grad, h_count, h_dtype, dtype, n_tensors, j0, 0);
      DW_HIP(pass == 0 ? launch_grad_squares(t, s) : launch_clip(t, s));
      t.part0 += t.chunks;
      t.out0 += t.elements;
    }
  }
  if (!writes) DW_HIP(launch_grad_norm(part, z.parts, d_norm, nullptr, k, s));
  return DW_OK;
}

int dw_fp8_quantize(const void* d_x, int64_t x_ld, int64_t x_stride, int k, int64_t rows, int64_t n, int dtype, int square,
                    uint8_t* d_q, uint8_t* d_scale, uint8_t* d_qt, uint8_t* d_scale_t, void* stream) {
  if (k < 1 || k > DW_MAX_K || !is_type(dtype)) return DW_ERR_CONFIG;
  if (rows < 0 || rows > DW_MAX_FP8 || n < 1 || n > DW_MAX_FP8 || (square != 0 && square != 1)) return DW_ERR_ARG;
  if (rows == 0) return DW_OK;                              // rows of the transposed matrix are empty too
  if (!d_x || (d_q && !d_scale) || (d_qt && !d_scale_t) || (!d_q && !d_qt)) return DW_ERR_NULL;
  if (!in_ok(d_x, x_ld, x_stride, rows, n, type_bytes(dtype))) return DW_ERR_ARG;
  if (!aligned(d_q, 16) || !aligned(d_qt, 16) || !aligned(d_scale, 4) || !aligned(d_scale_t, 4)) return DW_ERR_ARG;
  QuantArgs a = {};
  a.x = {d_x, x_ld, x_stride};
  a.k = k; a.square = square; a.rows = rows; a.n = n;
  a.q = d_q; a.scale = d_scale; a.qt = d_qt; a.scale_t = d_scale_t;
  DW_HIP(launch_fp8_quantize(a, dtype, (hipStream_t)stream));
  return DW_OK;
}

size_t dw_fp8_matmul_scratch_bytes(int k, int64_t m, int64_t n, int64_t contraction) {
  if (k < 1 || k > DW_MAX_K || m < 1 || m > DW_MAX_FP8 || n < 1 || n > DW_MAX_FP8 || contraction < 1 || contraction > DW_MAX_FP8) return 0;
  return fp8_scratch_bytes(k, m, n, DW_FP8_ROW(contraction));
}

int dw_fp8_matmul(const uint8_t* d_a, const uint8_t* d_a_scale, const uint8_t* d_b, const uint8_t* d_b_scale, const float* d_bias,
                  int64_t bias_stride, int k, int64_t m, int64_t n, int64_t contraction, int dtype, void* d_c, int64_t c_ld,
                  int64_t c_stride, void* d_scratch, size_t scratch_bytes, void* stream) {
  if (k < 1 || k > DW_MAX_K || !is_type(dtype)) return DW_ERR_CONFIG;
  if (m < 0 || m > DW_MAX_FP8 || n < 1 || n > DW_MAX_FP8 || contraction < 0 || contraction > DW_MAX_FP8) return DW_ERR_ARG;
  if (m == 0) return DW_OK;
  if (!d_c || (contraction > 0 && (!d_a || !d_a_scale || !d_b || !d_b_scale))) return DW_ERR_NULL;
  if (!aligned(d_a, 16) || !aligned(d_b, 16) || !aligned(d_a_scale, 4) || !aligned(d_b_scale, 4)) return DW_ERR_ARG;
  if (!params_ok(d_bias, bias_stride) || !out_ok(d_c, c_ld, c_stride, k, m, n, type_bytes(dtype))) return DW_ERR_ARG;
  if (!fp8_product_fits(k, m, n)) return DW_ERR_TOO_LARGE;
  const size_t need = dw_fp8_matmul_scratch_bytes(k, m, n, contraction);
  if (need > 0 && (!d_scratch || !aligned(d_scratch, 256) || scratch_bytes < need)) return DW_ERR_WORKSPACE;
  Fp8Args a = {};
  a.a = d_a; a.sa = d_a_scale; a.b = d_b; a.sb = d_b_scale;
  a.bias = d_bias; a.bias_stride = bias_stride;
  a.c = d_c; a.ldc = c_ld; a.c_stride = c_stride;
  a.k = k; a.dtype = dtype; a.m = m; a.n = n;
  a.kp = DW_FP8_ROW(contraction); a.ks = DW_FP8_SCALES(contraction);
  a.part = static_cast<float*>(d_scratch);
  DW_HIP(launch_fp8_matmul(a, (hipStream_t)stream));
  return DW_OK;
}

// scratch of dw_fp8_linear: x in 8 bits and its scales, and what the product needs; nothing where it is quantised on the way
static int64_t linear_q_bytes(int k, int64_t m, int64_t contraction) { return ceil_div(k * m * DW_FP8_ROW(contraction), 256) * 256; }
static int64_t linear_scale_bytes(int k, int64_t m, int64_t contraction) { return ceil_div(k * m * DW_FP8_SCALES(contraction), 256) * 256; }

size_t dw_fp8_linear_scratch_bytes(int k, int64_t m, int64_t n, int64_t contraction) {
  if (k < 1 || k > DW_MAX_K || m < 1 || m > DW_MAX_FP8 || n < 1 || n > DW_MAX_FP8 || contraction < 1 || contraction > DW_MAX_FP8) return 0;
  if (fp8_linear_fused(k, m, n, DW_FP8_ROW(contraction))) return 0;
  return (size_t)(linear_q_bytes(k, m, contraction) + linear_scale_bytes(k, m, contraction)) + dw_fp8_matmul_scratch_bytes(k, m, n, contraction);
}

int dw_fp8_linear(const void* d_x, int64_t x_ld, int64_t x_stride, const uint8_t* d_w, const uint8_t* d_w_scale, const float* d_bias,
                  int64_t bias_stride, int k, int64_t m, int64_t n, int64_t contraction, int dtype, void* d_y, int64_t y_ld,
                  int64_t y_stride, void* d_scratch, size_t scratch_bytes, void* stream) {
  if (k < 1 || k > DW_MAX_K || !is_type(dtype)) return DW_ERR_CONFIG;
  if (m < 0 || m > DW_MAX_FP8 || n < 1 || n > DW_MAX_FP8 || contraction < 1 || contraction > DW_MAX_FP8) return DW_ERR_ARG;
  if (m == 0) return DW_OK;
  if (!d_x || !d_w || !d_w_scale || !d_y) return DW_ERR_NULL;
  const int64_t b = type_bytes(dtype);
  if (!in_ok(d_x, x_ld, x_stride, m, contraction, b) || !aligned(d_w, 16) || !aligned(d_w_scale, 4)) return DW_ERR_ARG;
  if (!params_ok(d_bias, bias_stride) || !out_ok(d_y, y_ld, y_stride, k, m, n, b)) return DW_ERR_ARG;
  if (!fp8_product_fits(k, m, n)) return DW_ERR_TOO_LARGE;
  const size_t need = dw_fp8_linear_scratch_bytes(k, m, n, contraction);
  if (need > 0 && (!d_scratch || !aligned(d_scratch, 256) || scratch_bytes < need)) return DW_ERR_WORKSPACE;
  if (need == 0) {
    Fp8Args a = {};
    a.x = {d_x, x_ld, x_stride}; a.contraction = contraction;
    a.b = d_w; a.sb = d_w_scale;
    a.bias = d_bias; a.bias_stride = bias_stride;
    a.c = d_y; a.ldc = y_ld; a.c_stride = y_stride;
    a.k = k; a.dtype = dtype; a.m = m; a.n = n;
    a.kp = DW_FP8_ROW(contraction); a.ks = DW_FP8_SCALES(contraction);
    DW_HIP(launch_fp8_linear_fused(a, (hipStream_t)stream));
    return DW_OK;
  }
  uint8_t* q = static_cast<uint8_t*>(d_scratch);
  uint8_t* scale = q + linear_q_bytes(k, m, contraction);
  uint8_t* rest = scale + linear_scale_bytes(k, m, contraction);
  const int st = dw_fp8_quantize(d_x, x_ld, x_stride, k, m, contraction, dtype, 0, q, scale, nullptr, nullptr, stream);
  if (st != DW_OK) return st;
  return dw_fp8_matmul(q, scale, d_w, d_w_scale, d_bias, bias_stride, k, m, n, contraction, dtype, d_y, y_ld, y_stride, rest,
                       scratch_bytes - (size_t)(rest - q), stream);
}

}  // extern "C"
