// The routed-expert calls of libntc on torch tensors, for experts.py.
//
// A call of a serving step takes the GPU a few microseconds; checking tensors,
// allocating outputs and packing descriptors in Python took the host 9 to 23.  Each
// function here takes positional arguments (experts.py gives them names and
// defaults), checks its tensors, allocates its outputs and workspace with torch on
// the current stream and makes the one library call of its name.
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/Exceptions.h>

#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

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
                      "linear_backward and combine_backward compute it.");
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

#define ENTRY(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(route),           ENTRY(route_backward), ENTRY(expert_order),     ENTRY(linear),
                         ENTRY(linear_backward), ENTRY(combine),        ENTRY(combine_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_experts", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__experts() { return PyModule_Create(&module); }
