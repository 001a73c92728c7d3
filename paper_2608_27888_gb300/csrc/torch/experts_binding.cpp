// The routed-expert calls of libntc on torch tensors, for experts.py.
//
// A call of a serving step takes the GPU a few microseconds; checking tensors,
// allocating outputs and packing descriptors in Python took the host 9 to 23.  Each
// function here takes positional arguments (experts.py gives them names and
// defaults), checks its tensors, allocates its outputs and workspace with torch on
// the current stream and makes the one library call of its name.
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>

#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_strided.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include <memory>
#include <vector>

#include "ntc.h"

namespace {

using at::Tensor;

const Tensor &tensor(PyObject *o, const char *name) {
  TORCH_CHECK_TYPE(THPVariable_Check(o), name, " must be a tensor, not ", Py_TYPE(o)->tp_name);
  return THPVariable_Unpack(o);
}

// A result has no gradient, whatever its inputs ask for: said once, for a model would train on
// without it.
void not_recorded(std::initializer_list<PyObject *> inputs) {
  if (!at::GradMode::is_enabled()) return;
  for (PyObject *o : inputs)
    if (THPVariable_Check(o) && THPVariable_Unpack(o).requires_grad())
      TORCH_WARN_ONCE("autograd does not record route, linear and combine: their results have no gradient. route_backward, "
                      "linear_backward and combine_backward compute it. Nor does it record balance_loss, linear4, pack4 and unpack4.");
}

int64_t integer(PyObject *o, const char *name) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    TORCH_CHECK_TYPE(false, name, " must be an integer");
  }
  return v;
}
uint32_t small(PyObject *o, const char *name) {
  const int64_t v = integer(o, name);
  TORCH_CHECK_VALUE(v >= 0 && v <= 0xFFFFFFFFll, name, " is out of range: ", v);
  return (uint32_t)v;
}
float real(PyObject *o, const char *name) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    TORCH_CHECK_TYPE(false, name, " must be a number");
  }
  return (float)v;
}

// The device every tensor of a call is on: the current one.
void on_device(const Tensor &t, const char *name) {
  TORCH_CHECK_VALUE(t.is_cuda(), name, " must be a CUDA tensor");
  TORCH_CHECK_VALUE(t.get_device() == c10::cuda::current_device(), name, " is on ", t.device(),
                    ", which is not the current device");
}
ntc_type type_of(const Tensor &t, const char *name) {
  switch (t.scalar_type()) {
    case at::kFloat: return NTC_TYPE_FP32;
    case at::kHalf: return NTC_TYPE_FP16;
    case at::kBFloat16: return NTC_TYPE_BF16;
    default: TORCH_CHECK_VALUE(false, name, " must be float32, float16 or bfloat16, not ", t.scalar_type());
  }
}
void like(const Tensor &t, const char *name, at::ScalarType dtype, const Tensor &on) {
  TORCH_CHECK_VALUE(t.scalar_type() == dtype && t.device() == on.device(), name, " must be ", dtype, " on ", on.device(),
                    ", not ", t.scalar_type(), " on ", t.device());
}
void two_dims(const Tensor &t, const char *name) {
  TORCH_CHECK_VALUE(t.dim() == 2, name, " must have two dimensions, not ", t.dim());
}
// The row stride of a [rows, cols] matrix.
uint64_t matrix(const Tensor &t, const char *name, int64_t rows, int64_t cols, at::ScalarType dtype, const Tensor &on) {
  like(t, name, dtype, on);
  TORCH_CHECK_VALUE(t.dim() == 2 && t.size(0) == rows && t.size(1) == cols, name, " must have shape [", rows, ", ", cols,
                    "], not ", t.sizes());
  TORCH_CHECK_VALUE(cols <= 1 || t.stride(1) == 1, name, " must be contiguous along its last dimension");
  if (rows <= 1) return (uint64_t)cols;
  TORCH_CHECK_VALUE(t.stride(0) >= cols, name, " has overlapping rows");
  return (uint64_t)t.stride(0);
}
// The address of a contiguous array of this shape; None is null.
template <typename T>
const T *array(PyObject *o, const char *name, at::IntArrayRef shape, at::ScalarType dtype, const Tensor &on) {
  if (o == Py_None) return nullptr;
  const Tensor &t = tensor(o, name);
  like(t, name, dtype, on);
  TORCH_CHECK_VALUE(t.sizes() == shape, name, " must have shape ", shape, ", not ", t.sizes());
  TORCH_CHECK_VALUE(t.is_contiguous(), name, " must be contiguous");
  return (const T *)t.data_ptr();
}

Tensor fresh(at::IntArrayRef shape, at::ScalarType dtype, const Tensor &on) {
  return at::empty(shape, at::TensorOptions().dtype(dtype).device(on.device()));
}
void *stream_of(const Tensor &t) { return (void *)c10::cuda::getCurrentCUDAStream(t.get_device()).stream(); }
PyObject *wrap(const Tensor &t) { return THPVariable_Wrap(t); }
PyObject *wrap_or_none(const Tensor &t) {
  if (t.defined()) return wrap(t);
  Py_RETURN_NONE;
}
PyObject *tuple(std::initializer_list<PyObject *> items) {
  PyObject *r = PyTuple_New((Py_ssize_t)items.size());
  Py_ssize_t i = 0;
  for (PyObject *o : items) PyTuple_SET_ITEM(r, i++, o);
  return r;
}

// False, with NtcError raised, for a failed call.
bool done(ntc_status s) {
  if (s == NTC_OK) return true;
  PyObject *m = PyImport_ImportModule("paper_2608_27888_gb300.ntc");
  PyObject *cls = m ? PyObject_GetAttrString(m, "NtcError") : nullptr;
  if (cls) {
    PyObject *e = PyObject_CallFunction(cls, "is", (int)s, ntc_last_error());
    if (e) {
      PyErr_SetObject(cls, e);
      Py_DECREF(e);
    }
  }
  Py_XDECREF(cls);
  Py_XDECREF(m);
  return false;
}

bool takes(Py_ssize_t have, Py_ssize_t want) {
  if (have == want) return true;
  PyErr_Format(PyExc_TypeError, "%zd arguments are taken, %zd are given", want, have);
  return false;
}

// logits, top_k, bias, score, groups, top_groups, renormalize, scale -> ids, weights
PyObject *route(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!takes(n_args, 8)) return nullptr;
  not_recorded({a[0]});
  const Tensor &logits = tensor(a[0], "logits");
  on_device(logits, "logits");
  two_dims(logits, "logits");
  const int64_t n = logits.size(0), E = logits.size(1);
  ntc_route_desc d;
  d.num_experts = (uint32_t)std::min<int64_t>(E, 0xFFFFFFFFll);
  d.top_k = small(a[1], "top_k");
  d.score = small(a[3], "score");
  d.num_groups = small(a[4], "groups");
  d.top_groups = small(a[5], "top_groups");
  d.renormalize = small(a[6], "renormalize");
  d.scale = real(a[7], "scale");
  d.type = type_of(logits, "logits");
  const uint64_t ld = matrix(logits, "logits", n, E, logits.scalar_type(), logits);
  const float *bias = array<float>(a[2], "bias", {E}, at::kFloat, logits);
  TORCH_CHECK_VALUE(d.top_k <= NTC_MAX_TOP_K, "top_k must be in 1..min(32, num_experts)");
  Tensor ids = fresh({n, (int64_t)d.top_k}, at::kInt, logits), weights = fresh({n, (int64_t)d.top_k}, at::kFloat, logits);
  if (!done(ntc_route(&d, (size_t)n, logits.data_ptr(), ld, bias, (int32_t *)ids.data_ptr(), (float *)weights.data_ptr(),
                      stream_of(logits))))
    return nullptr;
  return tuple({wrap(ids), wrap(weights)});
  END_HANDLE_TH_ERRORS
}

// logits, ids, dweights, score, renormalize, scale -> dlogits
PyObject *route_backward(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!takes(n_args, 6)) return nullptr;
  const Tensor &logits = tensor(a[0], "logits"), &ids = tensor(a[1], "ids");
  on_device(logits, "logits");
  two_dims(logits, "logits");
  two_dims(ids, "ids");
  const int64_t n = logits.size(0), E = logits.size(1), k = ids.size(1);
  ntc_route_desc d;
  d.num_experts = (uint32_t)std::min<int64_t>(E, 0xFFFFFFFFll);
  d.top_k = (uint32_t)std::min<int64_t>(k, 0xFFFFFFFFll);
  d.num_groups = d.top_groups = 1;
  d.score = small(a[3], "score");
  d.renormalize = small(a[4], "renormalize");
  d.scale = real(a[5], "scale");
  d.type = type_of(logits, "logits");
  const uint64_t ld = matrix(logits, "logits", n, E, logits.scalar_type(), logits);
  const int32_t *i = array<int32_t>(a[1], "ids", {n, k}, at::kInt, logits);
  const float *g = array<float>(a[2], "dweights", {n, k}, at::kFloat, logits);
  Tensor out = fresh({n, E}, logits.scalar_type(), logits);
  if (!done(ntc_route_backward(&d, (size_t)n, logits.data_ptr(), ld, i, g, out.data_ptr(), stream_of(logits))))
    return nullptr;
  return wrap(out);
  END_HANDLE_TH_ERRORS
}

// ids, num_experts -> rows, place, offsets
PyObject *expert_order(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!takes(n_args, 2)) return nullptr;
  const Tensor &ids = tensor(a[0], "ids");
  on_device(ids, "ids");
  two_dims(ids, "ids");
  const int64_t n = ids.size(0), k = ids.size(1), E = integer(a[1], "num_experts");
  TORCH_CHECK_VALUE(E >= 1 && E <= NTC_MAX_EXPERTS, "num_experts must be in 1..", NTC_MAX_EXPERTS, ", not ", E);
  const int32_t *i = array<int32_t>(a[0], "ids", {n, k}, at::kInt, ids);
  Tensor rows = fresh({n * k}, at::kInt, ids), place = fresh({n, k}, at::kInt, ids), offsets = fresh({E + 1}, at::kInt, ids);
  const size_t size = ntc_expert_order_workspace((size_t)(n * k), (uint32_t)E);
  Tensor ws = size ? fresh({(int64_t)size}, at::kByte, ids) : Tensor();
  if (!done(ntc_expert_order(i, (size_t)(n * k), (uint32_t)std::min<int64_t>(k, 0xFFFFFFFFll), (uint32_t)E,
                             (int32_t *)rows.data_ptr(), (int32_t *)place.data_ptr(), (int32_t *)offsets.data_ptr(),
                             size ? ws.data_ptr() : nullptr, size, stream_of(ids))))
    return nullptr;
  return tuple({wrap(rows), wrap(place), wrap(offsets)});
  END_HANDLE_TH_ERRORS
}

// The descriptor of x and w ([E, N, K] or [N, K]) for `rows_out` rows.
ntc_linear_desc linear_desc(const Tensor &x, const Tensor &w, uint32_t activation, float slope, int64_t rows_out) {
  const int64_t dims = w.dim();
  TORCH_CHECK_VALUE(dims == 2 || dims == 3, "w must have two or three dimensions, not ", dims);
  const int64_t E = dims == 3 ? w.size(0) : 1, N = w.size(dims - 2), K = w.size(dims - 1);
  like(w, "w", x.scalar_type(), x);
  TORCH_CHECK_VALUE(K <= 1 || w.stride(dims - 1) == 1, "w must be contiguous along its last dimension");
  two_dims(x, "x");
  TORCH_CHECK_VALUE(E <= 0xFFFFFFFFll && N <= 0xFFFFFFFFll && K <= 0xFFFFFFFFll, "w is too large");
  ntc_linear_desc d;
  d.type = type_of(x, "x");
  d.in_dim = (uint32_t)K;
  d.out_dim = (uint32_t)N;
  d.num_experts = (uint32_t)E;
  d.activation = activation;
  d.leaky_slope = slope;
  d.num_rows = (uint64_t)rows_out;
  d.num_x_rows = (uint64_t)x.size(0);
  d.ld_x = matrix(x, "x", x.size(0), K, x.scalar_type(), x);
  d.ld_w = (uint64_t)(N > 1 ? w.stride(dims - 2) : K);
  d.stride_w = E > 1 ? (uint64_t)w.stride(0) : d.ld_w * (uint64_t)N;
  d.ld_y = d.ld_z = d.ld_residual = (uint64_t)N;
  return d;
}

// x, w, bias, rows, offsets, activation, leaky_slope, residual, save -> y, or (y, z)
PyObject *linear(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!takes(n_args, 9)) return nullptr;
  not_recorded({a[0], a[1], a[2], a[7]});
  const Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "w");
  on_device(x, "x");
  int64_t m = x.dim() ? x.size(0) : 0;
  if (a[3] != Py_None) {
    const Tensor &r = tensor(a[3], "rows");
    TORCH_CHECK_VALUE(r.dim() == 1, "rows must have one dimension, not ", r.dim());
    m = r.size(0);
  }
  ntc_linear_desc d = linear_desc(x, w, small(a[5], "activation"), real(a[6], "leaky_slope"), m);
  const int64_t E = d.num_experts, N = d.out_dim;
  const int32_t *rows = array<int32_t>(a[3], "rows", {m}, at::kInt, x);
  const int32_t *offsets = array<int32_t>(a[4], "offsets", {E + 1}, at::kInt, x);
  const float *bias = nullptr;
  if (a[2] != Py_None) {
    if (E == 1 && tensor(a[2], "bias").dim() == 1) bias = array<float>(a[2], "bias", {N}, at::kFloat, x);
    else bias = array<float>(a[2], "bias", {E, N}, at::kFloat, x);
  }
  const void *residual = nullptr;
  if (a[7] != Py_None) {
    const Tensor &r = tensor(a[7], "residual");
    d.ld_residual = matrix(r, "residual", m, N, x.scalar_type(), x);
    residual = r.data_ptr();
  }
  const bool save = PyObject_IsTrue(a[8]) == 1;
  const void *px = x.data_ptr(), *pw = w.data_ptr();
  Tensor y = fresh({m, N}, x.scalar_type(), x), z = save ? fresh({m, N}, x.scalar_type(), x) : Tensor();
  const size_t size = ntc_linear_workspace(&d, px, rows, pw);
  Tensor ws = size ? fresh({(int64_t)size}, at::kByte, x) : Tensor();
  if (!done(ntc_linear(&d, px, rows, offsets, pw, bias, residual, y.data_ptr(), save ? z.data_ptr() : nullptr,
                       size ? ws.data_ptr() : nullptr, size, stream_of(x))))
    return nullptr;
  return save ? tuple({wrap(y), wrap(z)}) : wrap(y);
  END_HANDLE_TH_ERRORS
}

// dy, x, w, z, rows, offsets, activation, leaky_slope, dx?, dw?, db? -> dx, dw, db
PyObject *linear_backward(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!takes(n_args, 11)) return nullptr;
  const Tensor &dy = tensor(a[0], "dy"), &x = tensor(a[1], "x"), &w = tensor(a[2], "w");
  on_device(x, "x");
  two_dims(dy, "dy");
  const int64_t m = dy.size(0);
  ntc_linear_desc d = linear_desc(x, w, small(a[6], "activation"), real(a[7], "leaky_slope"), m);
  const int64_t E = d.num_experts, N = d.out_dim, K = d.in_dim;
  const int32_t *rows = array<int32_t>(a[4], "rows", {m}, at::kInt, x);
  const int32_t *offsets = array<int32_t>(a[5], "offsets", {E + 1}, at::kInt, x);
  d.ld_y = matrix(dy, "dy", m, N, x.scalar_type(), x);
  const void *z = nullptr;
  if (d.activation != NTC_ACT_NONE) {
    TORCH_CHECK_VALUE(a[3] != Py_None, "an activation needs z");
    const Tensor &t = tensor(a[3], "z");
    d.ld_z = matrix(t, "z", m, N, x.scalar_type(), x);
    z = t.data_ptr();
  }
  const void *py = dy.data_ptr(), *px = x.data_ptr(), *pw = w.data_ptr();
  Tensor dx, dw, db;
  if (PyObject_IsTrue(a[8]) == 1) dx = fresh({m, K}, x.scalar_type(), x);
  if (PyObject_IsTrue(a[9]) == 1) dw = fresh(w.sizes(), x.scalar_type(), x);
  if (PyObject_IsTrue(a[10]) == 1) db = fresh(w.sizes().slice(0, (size_t)w.dim() - 1), at::kFloat, x);
  const size_t size = ntc_linear_backward_workspace(&d, py, px, rows, pw);
  Tensor ws = size ? fresh({(int64_t)size}, at::kByte, x) : Tensor();
  if (!done(ntc_linear_backward(&d, py, z, px, rows, offsets, pw, dx.defined() ? dx.data_ptr() : nullptr,
                                dw.defined() ? dw.data_ptr() : nullptr, db.defined() ? (float *)db.data_ptr() : nullptr,
                                size ? ws.data_ptr() : nullptr, size, stream_of(x))))
    return nullptr;
  return tuple({wrap_or_none(dx), wrap_or_none(dw), wrap_or_none(db)});
  END_HANDLE_TH_ERRORS
}

ntc_combine_desc combine_desc(const Tensor &y, const Tensor &place, PyObject *offsets) {
  on_device(y, "y");
  two_dims(y, "y");
  two_dims(place, "place");
  ntc_combine_desc d;
  d.type = type_of(y, "y");
  d.dim = (uint32_t)std::min<int64_t>(y.size(1), 0xFFFFFFFFll);
  d.top_k = (uint32_t)std::min<int64_t>(place.size(1), 0xFFFFFFFFll);
  d.num_experts = 1;
  if (offsets != Py_None) {
    const Tensor &o = tensor(offsets, "offsets");
    TORCH_CHECK_VALUE(o.dim() == 1 && o.size(0) >= 1, "offsets must have one dimension");
    d.num_experts = (uint32_t)std::min<int64_t>(o.size(0) - 1, 0xFFFFFFFFll);
  }
  d.num_tokens = (uint64_t)place.size(0);
  d.num_rows = (uint64_t)y.size(0);
  d.ld_y = matrix(y, "y", y.size(0), y.size(1), y.scalar_type(), y);
  d.ld_out = d.ld_residual = (uint64_t)y.size(1);
  return d;
}

// y, place, weights, offsets, residual -> out
PyObject *combine(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!takes(n_args, 5)) return nullptr;
  not_recorded({a[0], a[2], a[4]});
  const Tensor &y = tensor(a[0], "y"), &place = tensor(a[1], "place");
  ntc_combine_desc d = combine_desc(y, place, a[3]);
  const int64_t T = place.size(0), k = place.size(1), D = y.size(1);
  const int32_t *p = array<int32_t>(a[1], "place", {T, k}, at::kInt, y);
  const float *g = array<float>(a[2], "weights", {T, k}, at::kFloat, y);
  const int32_t *o = array<int32_t>(a[3], "offsets", {(int64_t)d.num_experts + 1}, at::kInt, y);
  const void *residual = nullptr;
  if (a[4] != Py_None) {
    const Tensor &r = tensor(a[4], "residual");
    d.ld_residual = matrix(r, "residual", T, D, y.scalar_type(), y);
    residual = r.data_ptr();
  }
  Tensor out = fresh({T, D}, y.scalar_type(), y);
  if (!done(ntc_combine(&d, y.data_ptr(), p, g, o, residual, out.data_ptr(), stream_of(y)))) return nullptr;
  return wrap(out);
  END_HANDLE_TH_ERRORS
}

// dout, y, place, weights, offsets, dy?, dweights? -> dy, dweights
PyObject *combine_backward(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!takes(n_args, 7)) return nullptr;
  const Tensor &dout = tensor(a[0], "dout"), &y = tensor(a[1], "y"), &place = tensor(a[2], "place");
  ntc_combine_desc d = combine_desc(y, place, a[4]);
  const int64_t T = place.size(0), k = place.size(1), D = y.size(1);
  const int32_t *p = array<int32_t>(a[2], "place", {T, k}, at::kInt, y);
  const float *g = array<float>(a[3], "weights", {T, k}, at::kFloat, y);
  const int32_t *o = array<int32_t>(a[4], "offsets", {(int64_t)d.num_experts + 1}, at::kInt, y);
  d.ld_out = matrix(dout, "dout", T, D, y.scalar_type(), y);
  Tensor dy, dw;
  if (PyObject_IsTrue(a[5]) == 1) dy = fresh({y.size(0), D}, y.scalar_type(), y);
  if (PyObject_IsTrue(a[6]) == 1) dw = fresh({T, k}, at::kFloat, y);
  if (!done(ntc_combine_backward(&d, dout.data_ptr(), y.data_ptr(), p, g, o, dy.defined() ? dy.data_ptr() : nullptr,
                                 dw.defined() ? (float *)dw.data_ptr() : nullptr, stream_of(y))))
    return nullptr;
  return tuple({wrap_or_none(dy), wrap_or_none(dw)});
  END_HANDLE_TH_ERRORS
}

ntc_balance_desc balance_desc(const Tensor &logits, const Tensor &ids, PyObject *score, PyObject *scale) {
  on_device(logits, "logits");
  two_dims(logits, "logits");
  two_dims(ids, "ids");
  ntc_balance_desc d;
  d.num_experts = (uint32_t)std::min<int64_t>(logits.size(1), 0xFFFFFFFFll);
  d.top_k = (uint32_t)std::min<int64_t>(ids.size(1), 0xFFFFFFFFll);
  d.score = small(score, "score");
  d.scale = real(scale, "scale");
  d.type = type_of(logits, "logits");
  return d;
}

// logits, ids, score, scale -> loss, counts, mean
PyObject *balance_loss(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!takes(n_args, 4)) return nullptr;
  not_recorded({a[0]});
  const Tensor &logits = tensor(a[0], "logits"), &ids = tensor(a[1], "ids");
  const ntc_balance_desc d = balance_desc(logits, ids, a[2], a[3]);
  const int64_t n = logits.size(0), E = logits.size(1);
  const uint64_t ld = matrix(logits, "logits", n, E, logits.scalar_type(), logits);
  const int32_t *i = array<int32_t>(a[1], "ids", {n, ids.size(1)}, at::kInt, logits);
  Tensor loss = fresh({}, at::kFloat, logits), counts = fresh({E + 1}, at::kInt, logits), mean = fresh({E}, at::kFloat, logits);
  const size_t size = ntc_balance_loss_workspace(&d, (size_t)n);
  Tensor ws = size ? fresh({(int64_t)size}, at::kByte, logits) : Tensor();
  if (!done(ntc_balance_loss(&d, (size_t)n, logits.data_ptr(), ld, i, (float *)loss.data_ptr(), (int32_t *)counts.data_ptr(),
                             (float *)mean.data_ptr(), size ? ws.data_ptr() : nullptr, size, stream_of(logits))))
    return nullptr;
  return tuple({wrap(loss), wrap(counts), wrap(mean)});
  END_HANDLE_TH_ERRORS
}

// The address of a tensor of one element; None is null.
template <typename T>
const T *scalar(PyObject *o, const char *name, at::ScalarType dtype, const Tensor &on) {
  if (o == Py_None) return nullptr;
  const Tensor &t = tensor(o, name);
  like(t, name, dtype, on);
  TORCH_CHECK_VALUE(t.numel() == 1, name, " must have one element, not ", t.numel());
  return (const T *)t.data_ptr();
}

// logits, ids, counts, dloss, residual, score, scale -> dlogits
PyObject *balance_loss_backward(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!takes(n_args, 7)) return nullptr;
  const Tensor &logits = tensor(a[0], "logits"), &ids = tensor(a[1], "ids");
  const ntc_balance_desc d = balance_desc(logits, ids, a[5], a[6]);
  const int64_t n = logits.size(0), E = logits.size(1);
  const uint64_t ld = matrix(logits, "logits", n, E, logits.scalar_type(), logits);
  const int32_t *i = array<int32_t>(a[1], "ids", {n, ids.size(1)}, at::kInt, logits);
  TORCH_CHECK_TYPE(a[2] != Py_None, "counts must be a tensor, not None");
  const int32_t *c = array<int32_t>(a[2], "counts", {E + 1}, at::kInt, logits);
  const float *g = scalar<float>(a[3], "dloss", at::kFloat, logits);
  const void *residual = nullptr;
  uint64_t ld_residual = (uint64_t)E;
  if (a[4] != Py_None) {
    const Tensor &r = tensor(a[4], "residual");
    ld_residual = matrix(r, "residual", n, E, logits.scalar_type(), logits);
    residual = r.data_ptr();
  }
  Tensor out = fresh({n, E}, logits.scalar_type(), logits);
  if (!done(ntc_balance_loss_backward(&d, (size_t)n, logits.data_ptr(), ld, i, c, g, residual, ld_residual, out.data_ptr(),
                                      stream_of(logits))))
    return nullptr;
  return wrap(out);
  END_HANDLE_TH_ERRORS
}

// The tensors of a sequence; an entry may be None where `optional`.
struct Tensors {
  PyObject *fast;
  const char *name;
  Tensors(PyObject *o, const char *n) : fast(PySequence_Fast(o, "")), name(n) {
    if (!fast) {
      PyErr_Clear();
      TORCH_CHECK_TYPE(false, name, " must be a sequence of tensors");
    }
  }
  Tensors(const Tensors &) = delete;
  ~Tensors() { Py_DECREF(fast); }
  Py_ssize_t size() const { return PySequence_Fast_GET_SIZE(fast); }
  bool none(Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(fast, i) == Py_None; }
  const Tensor &at(Py_ssize_t i) const { return tensor(PySequence_Fast_GET_ITEM(fast, i), name); }
  void as_many(Py_ssize_t n) const {
    TORCH_CHECK_VALUE(size() == n, name, " must have an entry for each parameter: ", n, ", not ", size());
  }
};
void same(const Tensor &t, const char *name, Py_ssize_t i, const Tensor &p) {
  TORCH_CHECK_VALUE(t.device() == p.device(), name, "[", i, "] is on ", t.device(), ", its parameter on ", p.device());
  TORCH_CHECK_VALUE(t.sizes() == p.sizes(), name, "[", i, "] must have shape ", p.sizes(), ", not ", t.sizes());
  TORCH_CHECK_VALUE(t.is_contiguous(), name, "[", i, "] must be contiguous");
}
void changed(const Tensor &t) {  // as an operation in place
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// params, grads, m, v, scales, copies, step, lr, beta1, beta2, eps, weight_decay, grad_scale -> None
PyObject *adamw(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!takes(n_args, 13)) return nullptr;
  const Tensors params(a[0], "params"), grads(a[1], "grads"), m(a[2], "m"), v(a[3], "v");
  const Py_ssize_t n = params.size();
  grads.as_many(n);
  m.as_many(n);
  v.as_many(n);
  std::unique_ptr<Tensors> scales, copies;
  if (a[4] != Py_None) scales.reset(new Tensors(a[4], "scales")), scales->as_many(n);
  if (a[5] != Py_None) copies.reset(new Tensors(a[5], "copies")), copies->as_many(n);
  ntc_adamw_desc d;
  const auto number = [](PyObject *o, const char *name) {
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) {
      PyErr_Clear();
      TORCH_CHECK_TYPE(false, name, " must be a number");
    }
    return x;
  };
  const bool t_step = THPVariable_Check(a[6]), t_lr = THPVariable_Check(a[7]), t_scale = THPVariable_Check(a[12]);
  int64_t step = 1;
  if (!t_step) step = integer(a[6], "step");
  TORCH_CHECK_VALUE(step >= 1, "step must be at least 1, not ", step);
  d.step = (uint64_t)step;
  d.lr = t_lr ? 0.0 : number(a[7], "lr");
  d.beta1 = number(a[8], "beta1");
  d.beta2 = number(a[9], "beta2");
  d.eps = number(a[10], "eps");
  d.weight_decay = number(a[11], "weight_decay");
  d.grad_scale = t_scale ? 1.0 : number(a[12], "grad_scale");
  if (n == 0) Py_RETURN_NONE;
  const bool eight = m.at(0).scalar_type() == at::kFloat8_e4m3fn;
  TORCH_CHECK_VALUE(eight == (bool)scales, eight ? "moments in float8_e4m3fn need scales" : "scales are for moments in float8_e4m3fn");
  d.moment_bits = eight ? 8 : 32;
  const at::ScalarType moments = eight ? at::kFloat8_e4m3fn : at::kFloat;
  const Tensor &first = params.at(0);
  on_device(first, "params[0]");
  std::vector<ntc_adamw_tensor> t((size_t)n);
  for (Py_ssize_t i = 0; i < n; ++i) {
    const Tensor &p = params.at(i), &g = grads.at(i), &mi = m.at(i), &vi = v.at(i);
    same(p, "params", i, p);
    TORCH_CHECK_VALUE(p.device() == first.device(), "params[", i, "] is on ", p.device(), ", params[0] on ", first.device());
    same(g, "grads", i, p);
    same(mi, "m", i, p);
    same(vi, "v", i, p);
    TORCH_CHECK_VALUE(mi.scalar_type() == moments && vi.scalar_type() == moments, "m[", i, "] and v[", i, "] must be ", moments,
                      " like m[0], not ", mi.scalar_type(), " and ", vi.scalar_type());
    ntc_adamw_tensor &x = t[(size_t)i];
    x.param = p.data_ptr();
    x.grad = g.data_ptr();
    x.m = mi.data_ptr();
    x.v = vi.data_ptr();
    x.scale_m = x.scale_v = nullptr;
    x.copy = nullptr;
    x.count = (uint64_t)p.numel();
    x.param_type = type_of(p, "a parameter");
    x.grad_type = type_of(g, "a gradient");
    x.copy_type = NTC_TYPE_FP32;
    if (eight) {
      const Tensor &s = scales->at(i);
      const int64_t blocks = (p.numel() + NTC_ADAMW_BLOCK - 1) / NTC_ADAMW_BLOCK;
      TORCH_CHECK_VALUE(s.scalar_type() == at::kFloat && s.device() == p.device() && s.dim() == 2 && s.size(0) == 2 && s.size(1) == blocks &&
                            (blocks <= 1 || s.stride(1) == 1),
                        "scales[", i, "] must be Float of shape [2, ", blocks, "] on ", p.device(), ", contiguous along the last dimension");
      x.scale_m = (float *)s.data_ptr();
      x.scale_v = x.scale_m + s.stride(0);
    }
    if (copies && !copies->none(i)) {
      const Tensor &c = copies->at(i);
      same(c, "copies", i, p);
      x.copy = c.data_ptr();
      x.copy_type = type_of(c, "a copy");
    }
  }
  const float *lr = t_lr ? scalar<float>(a[7], "lr", at::kFloat, first) : nullptr;
  const int32_t *count = t_step ? scalar<int32_t>(a[6], "step", at::kInt, first) : nullptr;
  const float *scale = t_scale ? scalar<float>(a[12], "grad_scale", at::kFloat, first) : nullptr;
  const bool device = lr || count || scale;
  Tensor ws = device ? fresh({(int64_t)NTC_ADAMW_WORKSPACE}, at::kByte, first) : Tensor();
  if (!done(ntc_adamw(&d, t.data(), (size_t)n, lr, count, scale, device ? ws.data_ptr() : nullptr, device ? NTC_ADAMW_WORKSPACE : 0,
                      stream_of(first))))
    return nullptr;
  for (Py_ssize_t i = 0; i < n; ++i) {
    changed(params.at(i));
    changed(m.at(i));
    changed(v.at(i));
    if (eight) changed(scales->at(i));
    if (t[(size_t)i].copy) changed(copies->at(i));
  }
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

// The strides of an array [E, N, cols] or [N, cols], in elements.
void rows_of(const Tensor &t, const char *name, int64_t E, int64_t N, int64_t cols, at::ScalarType dtype, const Tensor &on, uint64_t &ld,
             uint64_t &stride) {
  like(t, name, dtype, on);
  const int64_t dims = t.dim();
  TORCH_CHECK_VALUE((dims == 3 || (dims == 2 && E == 1)) && (dims == 2 || t.size(0) == E) && t.size(dims - 2) == N && t.size(dims - 1) == cols,
                    name, " must have shape [", E, ", ", N, ", ", cols, "], not ", t.sizes());
  TORCH_CHECK_VALUE(cols <= 1 || t.stride(dims - 1) == 1, name, " must be contiguous along its last dimension");
  ld = (uint64_t)(N > 1 ? t.stride(dims - 2) : cols);
  stride = E > 1 ? (uint64_t)t.stride(0) : ld * (uint64_t)N;
}
int64_t groups_of(int64_t K, uint32_t group) {
  TORCH_CHECK_VALUE(group == 32 || group == 64 || group == 128, "group must be 32, 64 or 128, not ", group);
  return (K + group - 1) / group;
}
// The descriptor of packed weights and their scales.
ntc_pack4_desc pack4_desc(const Tensor &packed, const Tensor &scales, int64_t K, uint32_t group) {
  const int64_t dims = packed.dim();
  TORCH_CHECK_VALUE(dims == 2 || dims == 3, "packed must have two or three dimensions, not ", dims);
  TORCH_CHECK_VALUE(K >= 1 && K <= 0xFFFFFFFFll, "d_in is out of range: ", K);
  const int64_t E = dims == 3 ? packed.size(0) : 1, N = packed.size(dims - 2);
  TORCH_CHECK_VALUE(E <= 0xFFFFFFFFll && N <= 0xFFFFFFFFll, "packed is too large");
  ntc_pack4_desc d;
  d.type = type_of(scales, "scales");
  d.in_dim = (uint32_t)K;
  d.out_dim = (uint32_t)N;
  d.num_experts = (uint32_t)E;
  d.group = group;
  rows_of(packed, "packed", E, N, (K + 1) / 2, at::kByte, packed, d.ld_packed, d.stride_packed);
  rows_of(scales, "scales", E, N, groups_of(K, group), scales.scalar_type(), packed, d.ld_scales, d.stride_scales);
  return d;
}

// w, group, dtype -> packed, scales
PyObject *pack4(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!takes(n_args, 3)) return nullptr;
  not_recorded({a[0]});
  const Tensor &w = tensor(a[0], "w");
  on_device(w, "w");
  const int64_t dims = w.dim();
  TORCH_CHECK_VALUE(dims == 2 || dims == 3, "w must have two or three dimensions, not ", dims);
  const int64_t E = dims == 3 ? w.size(0) : 1, N = w.size(dims - 2), K = w.size(dims - 1);
  const uint32_t group = small(a[1], "group");
  const ntc_type w_type = type_of(w, "w");
  at::ScalarType dtype = w_type == NTC_TYPE_FP32 ? at::kBFloat16 : w.scalar_type();
  if (a[2] != Py_None) {
    TORCH_CHECK_TYPE(THPDtype_Check(a[2]), "dtype must be a torch.dtype");
    dtype = ((THPDtype *)a[2])->scalar_type;
  }
  TORCH_CHECK_VALUE(dtype == at::kHalf || dtype == at::kBFloat16, "dtype must be float16 or bfloat16, not ", dtype);
  TORCH_CHECK_VALUE(E >= 1 && N >= 1 && K >= 1 && E <= 0xFFFFFFFFll && N <= 0xFFFFFFFFll && K <= 0xFFFFFFFFll, "w has shape ", w.sizes());
  uint64_t ld, stride;
  rows_of(w, "w", E, N, K, w.scalar_type(), w, ld, stride);
  const int64_t G = groups_of(K, group), bytes = (K + 1) / 2, pitch = (bytes + 15) / 16 * 16;
  std::vector<int64_t> shape = {N, bytes}, strides = {pitch, 1}, s_shape = {N, G};
  if (dims == 3) {
    shape.insert(shape.begin(), E);
    strides.insert(strides.begin(), N * pitch);
    s_shape.insert(s_shape.begin(), E);
  }
  Tensor packed = at::empty_strided(shape, strides, at::TensorOptions().dtype(at::kByte).device(w.device()));
  Tensor scales = fresh(s_shape, dtype, w);
  const ntc_pack4_desc d = pack4_desc(packed, scales, K, group);
  if (!done(ntc_pack4(&d, w.data_ptr(), w_type, ld, stride, (uint8_t *)packed.data_ptr(), scales.data_ptr(), stream_of(w)))) return nullptr;
  return tuple({wrap(packed), wrap(scales)});
  END_HANDLE_TH_ERRORS
}

// packed, scales, d_in, group -> w
PyObject *unpack4(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!takes(n_args, 4)) return nullptr;
  not_recorded({a[1]});
  const Tensor &packed = tensor(a[0], "packed"), &scales = tensor(a[1], "scales");
  on_device(packed, "packed");
  const int64_t K = integer(a[2], "d_in");
  const ntc_pack4_desc d = pack4_desc(packed, scales, K, small(a[3], "group"));
  std::vector<int64_t> shape = packed.sizes().vec();
  shape.back() = K;
  Tensor w = fresh(shape, scales.scalar_type(), packed);
  if (!done(ntc_unpack4(&d, (const uint8_t *)packed.data_ptr(), scales.data_ptr(), w.data_ptr(), (uint64_t)K,
                        (uint64_t)K * d.out_dim, stream_of(packed))))
    return nullptr;
  return wrap(w);
  END_HANDLE_TH_ERRORS
}

// x, packed, scales, bias, group, rows, offsets, activation, leaky_slope, residual -> y
PyObject *linear4(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!takes(n_args, 10)) return nullptr;
  not_recorded({a[0], a[2], a[3], a[9]});
  const Tensor &x = tensor(a[0], "x"), &packed = tensor(a[1], "packed"), &scales = tensor(a[2], "scales");
  on_device(x, "x");
  two_dims(x, "x");
  const int64_t K = x.size(1);
  like(packed, "packed", at::kByte, x);
  like(scales, "scales", x.scalar_type(), x);
  const ntc_pack4_desc p = pack4_desc(packed, scales, K, small(a[4], "group"));
  const int64_t E = p.num_experts, N = p.out_dim;
  int64_t m = x.size(0);
  if (a[5] != Py_None) {
    const Tensor &r = tensor(a[5], "rows");
    TORCH_CHECK_VALUE(r.dim() == 1, "rows must have one dimension, not ", r.dim());
    m = r.size(0);
  }
  ntc_linear_desc d;
  d.type = type_of(x, "x");
  d.in_dim = p.in_dim;
  d.out_dim = p.out_dim;
  d.num_experts = p.num_experts;
  d.activation = small(a[7], "activation");
  d.leaky_slope = real(a[8], "leaky_slope");
  d.num_rows = (uint64_t)m;
  d.num_x_rows = (uint64_t)x.size(0);
  d.ld_x = matrix(x, "x", x.size(0), K, x.scalar_type(), x);
  d.ld_w = d.stride_w = 0;
  d.ld_y = d.ld_z = d.ld_residual = (uint64_t)N;
  const int32_t *rows = array<int32_t>(a[5], "rows", {m}, at::kInt, x);
  const int32_t *offsets = array<int32_t>(a[6], "offsets", {E + 1}, at::kInt, x);
  const float *bias = nullptr;
  if (a[3] != Py_None) {
    if (E == 1 && tensor(a[3], "bias").dim() == 1) bias = array<float>(a[3], "bias", {N}, at::kFloat, x);
    else bias = array<float>(a[3], "bias", {E, N}, at::kFloat, x);
  }
  const void *residual = nullptr;
  if (a[9] != Py_None) {
    const Tensor &r = tensor(a[9], "residual");
    d.ld_residual = matrix(r, "residual", m, N, x.scalar_type(), x);
    residual = r.data_ptr();
  }
  Tensor y = fresh({m, N}, x.scalar_type(), x);
  const size_t size = ntc_linear4_workspace(&d, &p, x.data_ptr(), rows, (const uint8_t *)packed.data_ptr());
  Tensor ws = size ? fresh({(int64_t)size}, at::kByte, x) : Tensor();
  if (!done(ntc_linear4(&d, &p, x.data_ptr(), rows, offsets, (const uint8_t *)packed.data_ptr(), scales.data_ptr(), bias, residual,
                        y.data_ptr(), size ? ws.data_ptr() : nullptr, size, stream_of(x))))
    return nullptr;
  return wrap(y);
  END_HANDLE_TH_ERRORS
}

#define ENTRY(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(route),           ENTRY(route_backward), ENTRY(expert_order),     ENTRY(linear),
                         ENTRY(linear_backward), ENTRY(combine),        ENTRY(combine_backward), ENTRY(balance_loss),
                         ENTRY(balance_loss_backward), ENTRY(adamw),    ENTRY(pack4),            ENTRY(unpack4),
                         ENTRY(linear4),         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_experts", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__experts() { return PyModule_Create(&module); }
