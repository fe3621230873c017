// Tensor-level entry to the operators that need no handle: reads shapes, strides and addresses off torch tensors, allocates
// outputs and scratch on the current stream and calls the C functions of include/dw.h.  Host code only, a Python module of plain
// C functions with positional arguments; operators.py holds the documented signatures.
//
// It stands beside the ctypes binding because of what a call costs the caller: the smallest operators run 3 us on the GPU,
// and taking a tensor apart in Python costs 0.1 to 2 us for each property read (a layer norm 15 us a call, the clipping of
// 300 tensors 110).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <vector>

#include "dw.h"

namespace {

PyObject* g_error = nullptr;          // binding.DwError
PyObject* g_raw_stream = nullptr;     // torch._C._cuda_getCurrentRawStream

// ---- arguments -------------------------------------------------------------------------------------------------------

const at::Tensor& tensor(PyObject* o, const char* name) {
  TORCH_CHECK_VALUE(THPVariable_Check(o), name, " is no tensor");
  return THPVariable_Unpack(o);
}
const at::Tensor* maybe(PyObject* o, const char* name) { return o == Py_None ? nullptr : &tensor(o, name); }

double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw python_error();
  return v;
}
int64_t whole(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  return (int64_t)v;
}

int type_of(const at::Tensor& t, const char* name) {
  const at::ScalarType s = t.scalar_type();
  TORCH_CHECK_VALUE(s == at::kFloat || s == at::kBFloat16, name, " has type ", s, ": float32 or bfloat16 is wanted");
  return s == at::kBFloat16 ? DW_BF16 : DW_F32;
}

bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw python_error();
  return v != 0;
}

struct Matrix { void* p; int64_t ld, stride; };

// a [k][rows][n] tensor with contiguous rows
Matrix matrix(const at::Tensor& t, const char* name) {
  TORCH_CHECK_VALUE(t.dim() == 3, name, " has shape ", t.sizes(), ": [k][rows][n] is wanted");
  const int64_t k = t.size(0), rows = t.size(1), n = t.size(2);
  TORCH_CHECK_VALUE(n <= 1 || t.stride(2) == 1, "the rows of ", name, " are not contiguous");
  const int64_t ld = rows <= 1 ? n : t.stride(1);
  return {t.data_ptr(), ld, k <= 1 ? rows * ld : t.stride(0)};
}
Matrix matrix_like(const at::Tensor& t, const char* name, at::IntArrayRef shape, at::ScalarType type, at::Device device) {
  TORCH_CHECK_VALUE(t.sizes() == shape && t.scalar_type() == type && t.device() == device, name, " is ", t.scalar_type(), " ", t.sizes(),
                    " on ", t.device(), ": ", type, " ", shape, " on ", device, " is wanted");
  return matrix(t, name);
}

struct Param { float* p; int64_t stride; };
// float32 [k][n] with contiguous rows, such as a view of flat parameter vectors
Param param(const at::Tensor* t, const char* name, int64_t k, int64_t n, at::Device device) {
  if (!t) return {nullptr, n};
  TORCH_CHECK_VALUE(t->dim() == 2 && t->size(0) == k && t->size(1) == n && t->scalar_type() == at::kFloat && t->device() == device, name, " is ",
                    t->scalar_type(), " ", t->sizes(), " on ", t->device(), ": float32 [", k, "][", n, "] on ", device, " is wanted");
  TORCH_CHECK_VALUE(n <= 1 || t->stride(1) == 1, "the rows of ", name, " are not contiguous");
  return {static_cast<float*>(t->data_ptr()), k == 1 ? n : t->stride(0)};
}

// a contiguous [k][rows] tensor
void* values(const at::Tensor* t, const char* name, int64_t k, int64_t rows, at::ScalarType type, at::Device device) {
  if (!t) return nullptr;
  TORCH_CHECK_VALUE(t->dim() == 2 && t->size(0) == k && t->size(1) == rows && t->scalar_type() == type && t->device() == device && t->is_contiguous(),
                    name, " is ", t->scalar_type(), " ", t->sizes(), " on ", t->device(), ": a contiguous ", type, " [", k, "][", rows, "] on ", device, " is wanted");
  return t->data_ptr();
}

// the device's current stream; the guard makes the device the current one for the launches
struct On {
  void* stream;
  c10::DeviceGuard guard;
  static at::Device checked(const at::Tensor& t) {
    TORCH_CHECK_VALUE(t.is_cuda(), "tensors on a GPU are wanted: got ", t.device());
    return t.device();
  }
  explicit On(const at::Tensor& t) : guard(checked(t)) {
    PyObject* index = PyLong_FromLong(t.get_device());
    PyObject* s = index ? PyObject_CallOneArg(g_raw_stream, index) : nullptr;
    Py_XDECREF(index);
    if (!s) throw python_error();
    stream = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    if (PyErr_Occurred()) throw python_error();
  }
};

// straight from the device's allocator: the way through at::empty takes longer than a small call's launch has to spare
at::Tensor make(at::IntArrayRef shape, at::ScalarType type, at::Device device) { return at::detail::empty_cuda(shape, type, device, std::nullopt); }

// scratch that torch hands out again only to work behind this call's on the same stream
struct Scratch {
  at::Tensor t;
  void* p = nullptr;
  size_t bytes;
  Scratch(size_t n, at::Device device) : bytes(n) {
    if (n == 0) return;
    t = make({(int64_t)n}, at::kByte, device);
    if (reinterpret_cast<uintptr_t>(t.data_ptr()) % 256) t = make({(int64_t)n + 256}, at::kByte, device);
    p = reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(t.data_ptr()) + 255) / 256 * 256);
  }
};

void check(int status, const char* where) {
  if (status >= 0) return;
  PyObject* args = Py_BuildValue("(is)", status, where);
  if (args) {
    PyErr_SetObject(g_error, args);
    Py_DECREF(args);
  }
  throw python_error();
}

// a tensor of the caller's has been written to: a graph of autograd's that saved it sees that its values are gone, as it does
// behind torch's own in-place operators (tensors made in inference mode have no versions, and no graph saves them)
void written(PyObject* o) {
  if (o == Py_None) return;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

int workers_of(int64_t k) {                                  // (what does not fit an int is refused as too many)
  return k > DW_MAX_K ? DW_MAX_K + 1 : (int)k;
}

PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }
PyObject* none() { Py_RETURN_NONE; }
PyObject* wrap_or_none(const at::Tensor& t) { return t.defined() ? wrap(t) : none(); }

template <class... T>
PyObject* tuple(T... objects) {                              // takes the references
  PyObject* items[] = {objects...};
  for (PyObject* o : items)
    if (!o) throw python_error();
  PyObject* r = PyTuple_New(sizeof...(objects));
  if (!r) throw python_error();
  Py_ssize_t i = 0;
  for (PyObject* o : items) PyTuple_SET_ITEM(r, i++, o);
  return r;
}

void expect(Py_ssize_t got, Py_ssize_t want) { TORCH_CHECK_VALUE(got == want, "takes ", want, " arguments, got ", got); }

// ---- layer norm ------------------------------------------------------------------------------------------------------

// x, gamma, beta, eps, out, stats -> (y, mean, rstd)
PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  expect(n_args, 6);
  const at::Tensor& x = tensor(a[0], "x");
  const int type = type_of(x, "x");
  const Matrix mx = matrix(x, "x");
  const int64_t k = x.size(0), rows = x.size(1), n = x.size(2);
  On on(x);
  const at::Tensor* gamma = maybe(a[1], "gamma");
  const at::Tensor* beta = maybe(a[2], "beta");
  const Param g = param(gamma, "gamma", k, n, x.device()), b = param(beta, "beta", k, n, x.device());
  TORCH_CHECK_VALUE(!gamma || !beta || g.stride == b.stride, "gamma and beta have different worker strides");
  const double eps = number(a[3]);
  const at::Tensor y = a[4] == Py_None ? make(x.sizes(), x.scalar_type(), x.device()) : tensor(a[4], "out");
  const Matrix my = matrix_like(y, "out", x.sizes(), x.scalar_type(), x.device());
  at::Tensor mean, rstd;
  if (truth(a[5])) {
    mean = make({k, rows}, at::kFloat, x.device());
    rstd = make({k, rows}, at::kFloat, x.device());
  }
  check(dw_layer_norm(mx.p, mx.ld, mx.stride, g.p, b.p, gamma ? g.stride : b.stride, workers_of(k), rows, n, type, (float)eps, my.p, my.ld,
                      my.stride, mean.defined() ? static_cast<float*>(mean.data_ptr()) : nullptr,
                      rstd.defined() ? static_cast<float*>(rstd.data_ptr()) : nullptr, on.stream),
        "dw_layer_norm");
  written(a[4]);
  return tuple(wrap(y), wrap_or_none(mean), wrap_or_none(rstd));
  END_HANDLE_TH_ERRORS
}

// dy, x, gamma, mean, rstd, dx, dgamma, dbeta, want_dx, want_params -> (dx, dgamma, dbeta)
PyObject* layer_norm_grad(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  expect(n_args, 10);
  const at::Tensor& x = tensor(a[1], "x");
  const int type = type_of(x, "x");
  const Matrix mx = matrix(x, "x");
  const int64_t k = x.size(0), rows = x.size(1), n = x.size(2);
  On on(x);
  const Matrix mdy = matrix_like(tensor(a[0], "dy"), "dy", x.sizes(), x.scalar_type(), x.device());
  const Param g = param(maybe(a[2], "gamma"), "gamma", k, n, x.device());
  const void* mean = values(&tensor(a[3], "mean"), "mean", k, rows, at::kFloat, x.device());
  const void* rstd = values(&tensor(a[4], "rstd"), "rstd", k, rows, at::kFloat, x.device());
  at::Tensor dx, dgamma, dbeta;
  Matrix mdx = {nullptr, n, rows * n};
  if (truth(a[8])) {
    dx = a[5] == Py_None ? make(x.sizes(), x.scalar_type(), x.device()) : tensor(a[5], "dx");
    mdx = matrix_like(dx, "dx", x.sizes(), x.scalar_type(), x.device());
  }
  Param dg = {nullptr, n}, db = {nullptr, n};
  at::Tensor through;                                        // [k][n] for the one that is given, where the other has no layout of its own
  if (truth(a[9])) {
    dgamma = a[6] == Py_None ? make({k, n}, at::kFloat, x.device()) : tensor(a[6], "dgamma");
    dbeta = a[7] == Py_None ? make({k, n}, at::kFloat, x.device()) : tensor(a[7], "dbeta");
    dg = param(&dgamma, "dgamma", k, n, x.device());
    db = param(&dbeta, "dbeta", k, n, x.device());
    if (dg.stride != db.stride) {
      TORCH_CHECK_VALUE(a[6] == Py_None || a[7] == Py_None, "dgamma and dbeta have different worker strides");
      TORCH_CHECK_VALUE(dg.stride >= n && db.stride >= n, "the workers' rows of ", a[6] == Py_None ? "dbeta" : "dgamma", " overlap");
      through = make({k, n}, at::kFloat, x.device());
      (a[6] == Py_None ? db : dg) = param(&through, "dgamma", k, n, x.device());
    }
  }
  const Scratch scratch(dg.p ? dw_layer_norm_grad_scratch_bytes(workers_of(k), rows, n, type) : 0, x.device());
  check(dw_layer_norm_grad(mdy.p, mdy.ld, mdy.stride, mx.p, mx.ld, mx.stride, g.p, g.stride, static_cast<const float*>(mean),
                           static_cast<const float*>(rstd), workers_of(k), rows, n, type, mdx.p, mdx.ld, mdx.stride, dg.p, db.p, dg.stride,
                           scratch.p, scratch.bytes, on.stream),
        "dw_layer_norm_grad");
  if (through.defined()) {
    at::AutoDispatchBelowADInplaceOrView below;               // (written() below counts it, and autograd has no part in it)
    (a[6] == Py_None ? dbeta : dgamma).copy_(through);
  }
  if (dx.defined()) written(a[5]);
  if (dg.p) { written(a[6]); written(a[7]); }
  return tuple(wrap_or_none(dx), wrap_or_none(dgamma), wrap_or_none(dbeta));
  END_HANDLE_TH_ERRORS
}

// ---- policy loss -----------------------------------------------------------------------------------------------------

// logits, target, out -> logp
PyObject* token_logp(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  expect(n_args, 3);
  const at::Tensor& z = tensor(a[0], "logits");
  const int type = type_of(z, "logits");
  const Matrix mz = matrix(z, "logits");
  const int64_t k = z.size(0), rows = z.size(1), vocab = z.size(2);
  On on(z);
  const void* target = values(&tensor(a[1], "target"), "target", k, rows, at::kInt, z.device());
  const at::Tensor out = a[2] == Py_None ? make({k, rows}, at::kFloat, z.device()) : tensor(a[2], "out");
  void* po = values(&out, "out", k, rows, at::kFloat, z.device());
  check(dw_token_logp(mz.p, mz.ld, mz.stride, static_cast<const int32_t*>(target), workers_of(k), rows, vocab, type, static_cast<float*>(po),
                      on.stream),
        "dw_token_logp");
  written(a[2]);
  return wrap(out);
  END_HANDLE_TH_ERRORS
}

// logits, target, old_logp, advantage, weight, ref_logp, clip_low, clip_high, kl_coef, grad, want_grad -> (loss, logp, grad)
PyObject* policy_loss(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  expect(n_args, 11);
  const at::Tensor& z = tensor(a[0], "logits");
  const int type = type_of(z, "logits");
  const Matrix mz = matrix(z, "logits");
  const int64_t k = z.size(0), rows = z.size(1), vocab = z.size(2);
  On on(z);
  const void* target = values(&tensor(a[1], "target"), "target", k, rows, at::kInt, z.device());
  const char* names[] = {"old_logp", "advantage", "weight", "ref_logp"};
  const float* row[4];
  for (int i = 0; i < 4; ++i) {
    TORCH_CHECK_VALUE(i >= 2 || a[2 + i] != Py_None, names[i], " is wanted");
    row[i] = static_cast<const float*>(values(maybe(a[2 + i], names[i]), names[i], k, rows, at::kFloat, z.device()));
  }
  const double low = number(a[6]), high = number(a[7]), kl = number(a[8]);
  at::Tensor grad;
  Matrix mg = {nullptr, vocab, rows * vocab};
  if (truth(a[10])) {
    grad = a[9] == Py_None ? make(z.sizes(), z.scalar_type(), z.device()) : tensor(a[9], "grad");
    mg = matrix_like(grad, "grad", z.sizes(), z.scalar_type(), z.device());
  }
  const at::Tensor loss = make({k}, at::kFloat, z.device()), logp = make({k, rows}, at::kFloat, z.device());
  const Scratch scratch(dw_policy_loss_scratch_bytes(workers_of(k), rows), z.device());
  check(dw_policy_loss(mz.p, mz.ld, mz.stride, static_cast<const int32_t*>(target), row[0], row[3], row[1], row[2], workers_of(k), rows, vocab,
                       type, (float)low, (float)high, (float)kl, static_cast<float*>(loss.data_ptr()), static_cast<float*>(logp.data_ptr()),
                       mg.p, mg.ld, mg.stride, scratch.p, scratch.bytes, on.stream),
        "dw_policy_loss");
  if (grad.defined()) written(a[9]);
  return tuple(wrap(loss), wrap(logp), wrap_or_none(grad));
  END_HANDLE_TH_ERRORS
}

// ---- gradient norm and clipping --------------------------------------------------------------------------------------

// grads (a list or tuple), max_norm, workers, out -> norms
PyObject* clip_grads(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  expect(n_args, 4);
  PyObject* list = PySequence_Fast(a[0], "a sequence of tensors is wanted");
  if (!list) throw python_error();
  struct Release { PyObject* o; ~Release() { Py_DECREF(o); } } release{list};
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(list);
  PyObject** items = PySequence_Fast_ITEMS(list);
  const double max_norm = number(a[1]);
  const int64_t workers = whole(a[2]);
  TORCH_CHECK_VALUE(n > 0, "no tensors");
  TORCH_CHECK_VALUE(workers >= 1 && n % workers == 0, n, " tensors for ", workers, " workers");
  const Py_ssize_t per = n / workers;
  const at::Tensor& first = tensor(items[0], "a gradient");
  On on(first);
  std::vector<const void*> address(n);
  std::vector<int64_t> count(per);
  std::vector<int32_t> type(per);
  int64_t total = 0;
  for (Py_ssize_t i = 0, j = 0; i < n; ++i, j = j + 1 < per ? j + 1 : 0) {
    const at::Tensor& g = tensor(items[i], "a gradient");
    TORCH_CHECK_VALUE(g.device() == first.device(), "gradients on ", first.device(), " and ", g.device());
    TORCH_CHECK_VALUE(g.is_contiguous(), "a gradient is not contiguous");
    const int32_t t = type_of(g, "a gradient");
    address[i] = g.data_ptr();
    if (i < per) {
      count[i] = g.numel();
      type[i] = t;
      total += count[i];
    } else {
      TORCH_CHECK_VALUE(count[j] == g.numel() && type[j] == t, "worker ", i / per, " has tensors of other sizes or types than worker 0");
    }
  }
  const Param out = param(maybe(a[3], "out"), "out", workers, total, first.device());
  const at::Tensor norm = make({workers}, at::kFloat, first.device());
  const int k = workers_of(workers), tensors = per > DW_MAX_TENSORS ? DW_MAX_TENSORS + 1 : (int)per;
  const Scratch scratch(dw_clip_grads_scratch_bytes(k, tensors, count.data()), first.device());
  check(dw_clip_grads(address.data(), count.data(), type.data(), k, tensors, DW_F32, (float)max_norm, out.p, out.stride,
                      static_cast<float*>(norm.data_ptr()), scratch.p, scratch.bytes, on.stream),
        "dw_clip_grads");
  written(a[3]);
  if (!out.p && std::isfinite((float)max_norm))
    for (Py_ssize_t i = 0; i < n; ++i) written(items[i]);
  return wrap(norm);
  END_HANDLE_TH_ERRORS
}

// ---- products in 8 bits ----------------------------------------------------------------------------------------------

struct Eight { at::Tensor q, scale; };

Eight make_eight(int64_t k, int64_t rows, int64_t n, at::Device device) {
  return {make({k, rows, DW_FP8_ROW(n)}, at::kFloat8_e4m3fn, device), make({k, rows, DW_FP8_SCALES(n)}, at::kByte, device)};
}
uint8_t* bytes(const at::Tensor& t) { return t.defined() ? static_cast<uint8_t*>(t.data_ptr()) : nullptr; }

// x, square, transposed -> (q, scale) or (q, scale, qt, scale_t)
PyObject* fp8_quantize(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  expect(n_args, 3);
  const at::Tensor& x = tensor(a[0], "x");
  const int type = type_of(x, "x");
  const Matrix mx = matrix(x, "x");
  On on(x);
  const int64_t k = x.size(0), rows = x.size(1), n = x.size(2);
  const Eight m = make_eight(k, rows, n, x.device());
  Eight t;
  if (truth(a[2])) t = make_eight(k, n, rows, x.device());
  check(dw_fp8_quantize(mx.p, mx.ld, mx.stride, workers_of(k), rows, n, type, truth(a[1]) ? 1 : 0, bytes(m.q), bytes(m.scale), bytes(t.q),
                        bytes(t.scale), on.stream),
        "dw_fp8_quantize");
  if (t.q.defined()) return tuple(wrap(m.q), wrap(m.scale), wrap(t.q), wrap(t.scale));
  return tuple(wrap(m.q), wrap(m.scale));
  END_HANDLE_TH_ERRORS
}

// the operands of a product as an Fp8Matrix holds them: numbers, scales, length of a row
Eight operand(PyObject* q, PyObject* scale, int64_t n, const char* name) {
  const Eight e = {tensor(q, name), tensor(scale, name)};
  TORCH_CHECK_VALUE(n >= 0 && e.q.dim() == 3 && e.scale.dim() == 3 && e.q.scalar_type() == at::kFloat8_e4m3fn && e.scale.scalar_type() == at::kByte &&
                    e.q.size(2) == DW_FP8_ROW(n) && e.scale.size(2) == DW_FP8_SCALES(n) && e.q.size(0) == e.scale.size(0) &&
                    e.q.size(1) == e.scale.size(1) && e.q.is_contiguous() && e.scale.is_contiguous() && e.q.device() == e.scale.device(),
                    name, " is no matrix in 8 bits with rows of ", n);
  return e;
}

// a's numbers, scales, row length, b's, bias, out, bf16 -> c
PyObject* fp8_matmul(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  expect(n_args, 9);
  const int64_t n = whole(a[2]);
  TORCH_CHECK_VALUE(n == whole(a[5]), "operands with rows of ", n, " and ", whole(a[5]));
  const Eight x = operand(a[0], a[1], n, "a"), w = operand(a[3], a[4], n, "b");
  On on(x.q);
  const at::Device device = x.q.device();
  const int64_t k = x.q.size(0), m = x.q.size(1), rows = w.q.size(1);
  TORCH_CHECK_VALUE(w.q.size(0) == k && w.q.device() == device, "operands of ", k, " workers on ", device, " and ", w.q.size(0), " on ", w.q.device());
  const Param b = param(maybe(a[6], "bias"), "bias", k, rows, device);
  const at::Tensor c = a[7] == Py_None ? make({k, m, rows}, truth(a[8]) ? at::kBFloat16 : at::kFloat, device) : tensor(a[7], "out");
  const int code = type_of(c, "out");
  const Matrix mc = matrix_like(c, "out", {k, m, rows}, c.scalar_type(), device);
  const Scratch scratch(dw_fp8_matmul_scratch_bytes(workers_of(k), m, rows, n), device);
  check(dw_fp8_matmul(bytes(x.q), bytes(x.scale), bytes(w.q), bytes(w.scale), b.p, b.stride, workers_of(k), m, rows, n, code, mc.p, mc.ld,
                      mc.stride, scratch.p, scratch.bytes, on.stream),
        "dw_fp8_matmul");
  written(a[7]);
  return wrap(c);
  END_HANDLE_TH_ERRORS
}

// x, the weight's numbers, scales, row length, bias, out -> y
PyObject* fp8_linear(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  expect(n_args, 6);
  const at::Tensor& x = tensor(a[0], "x");
  const int type = type_of(x, "x");
  const Matrix mx = matrix(x, "x");
  On on(x);
  const at::Device device = x.device();
  const int64_t n = whole(a[3]), k = x.size(0), m = x.size(1);
  TORCH_CHECK_VALUE(x.size(2) == n, "x has rows of ", x.size(2), ", the weight of ", n);
  const Eight w = operand(a[1], a[2], n, "the weight");
  const int64_t rows = w.q.size(1);
  TORCH_CHECK_VALUE(w.q.size(0) == k && w.q.device() == device, "x of ", k, " workers on ", device, ", a weight of ", w.q.size(0), " on ", w.q.device());
  const Param b = param(maybe(a[4], "bias"), "bias", k, rows, device);
  const at::Tensor y = a[5] == Py_None ? make({k, m, rows}, x.scalar_type(), device) : tensor(a[5], "out");
  const Matrix my = matrix_like(y, "out", {k, m, rows}, x.scalar_type(), device);
  const Scratch scratch(dw_fp8_linear_scratch_bytes(workers_of(k), m, rows, n), device);
  check(dw_fp8_linear(mx.p, mx.ld, mx.stride, bytes(w.q), bytes(w.scale), b.p, b.stride, workers_of(k), m, rows, n, type, my.p, my.ld, my.stride,
                      scratch.p, scratch.bytes, on.stream),
        "dw_fp8_linear");
  written(a[5]);
  return wrap(y);
  END_HANDLE_TH_ERRORS
}

// the class of errors for a negative status
PyObject* set_error(PyObject*, PyObject* cls) {
  Py_INCREF(cls);
  Py_XDECREF(g_error);
  g_error = cls;
  Py_RETURN_NONE;
}

#define DW_FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {DW_FAST(layer_norm), DW_FAST(layer_norm_grad), DW_FAST(token_logp), DW_FAST(policy_loss), DW_FAST(clip_grads),
                         DW_FAST(fp8_quantize), DW_FAST(fp8_matmul), DW_FAST(fp8_linear), {"set_error", set_error, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_dw_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__dw_torch(void) {
  PyObject* c = PyImport_ImportModule("torch._C");
  if (!c) return nullptr;
  g_raw_stream = PyObject_GetAttrString(c, "_cuda_getCurrentRawStream");
  Py_DECREF(c);
  if (!g_raw_stream) return nullptr;
  Py_INCREF(PyExc_RuntimeError);
  g_error = PyExc_RuntimeError;
  return PyModule_Create(&module);
}
