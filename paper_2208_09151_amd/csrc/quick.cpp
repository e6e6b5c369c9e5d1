// The calls of the layers' Python names for the plain case, without the interpreter's part: tensors' descriptors are made and
// outputs allocated here.  Every function gives None for whatever it does not take (tensors elsewhere, other types or shapes, a
// gradient that is to be recorded, a tangent of forward mode, tensors with a __torch_dispatch__ of their own), and the Python names
// go on with what they do without it; nothing is refused here.  The call's status comes with the result, for the Python name to
// raise what the library says.
//
// Measured on the host, us of a call without and with it: linear 12.8 and 5.3, expert_layer 15.2 and 7.8, layer norm 10.6 and 5.2, its
// gradients 16.9 and 9.5, lookup 8.1 and 4.1, its gradient 23.7 and 19.1 (a dozen launches).
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/AutogradState.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/autograd/python_variable.h>

#include "ginex_layers.h"

// What this is compiled against; the Python side looks for it in the file before it loads it.
extern "C" __attribute__((used, visibility("default"))) const char ginex_quick_is_for[] = GINEX_QUICK_IS_FOR;

namespace {

// A tensor that carries a tangent of forward mode (there is one level of those).
bool has_tangent(const at::Tensor& t) { return c10::AutogradState::get_tls_state().get_fw_grad_mode() && t._fw_grad(0).defined(); }

// A tensor that is used as it is: in the memory of GPU `device`, with no gradient to record.
bool plain(PyObject* o, int device, at::Tensor& t) {
  if (!THPVariable_Check(o)) return false;
  t = THPVariable_Unpack(o);
  return t.is_cuda() && t.get_device() == device && t.layout() == at::kStrided && !t.key_set().has(c10::DispatchKey::Python) &&
         !t.is_neg() && !(t.requires_grad() && c10::GradMode::is_enabled()) && !has_tangent(t);
}

// Other threads run while the library does.
struct Unlocked {
  PyThreadState* const state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <typename Call>
int32_t unlocked(Call call) {
  const Unlocked now;
  return call();
}

int32_t type_of(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return GINEX_F32;
    case at::kBFloat16: return GINEX_BF16;
    case at::kHalf: return GINEX_F16;
    default: return -1;
  }
}

bool rows_of(const at::Tensor& t, ginex_rows_t& r) {
  if (t.dim() != 2) return false;
  const int32_t type = type_of(t);
  const int64_t n = t.size(0), width = t.size(1);
  if (type < 0 || (t.stride(1) != 1 && width > 1)) return false;
  r = {t.data_ptr(), n, width, n <= 1 ? width : t.stride(0), type};
  return true;
}

bool weights_of(const at::Tensor& t, int64_t dims, at::ScalarType type, ginex_weights_t& w) {
  if (t.dim() != dims || t.scalar_type() != type) return false;
  const int64_t width = t.size(dims - 2), out = t.size(dims - 1), along = t.stride(dims - 2), across = t.stride(dims - 1);
  int32_t turned;
  int64_t stride;
  if (across == 1 || out == 1) {
    turned = 0;
    stride = width == 1 ? out : along;
  } else if (along == 1 || width == 1) {
    turned = 1;
    stride = across;
  } else {
    return false;
  }
  const int64_t experts = dims == 3 ? t.size(0) : 1;
  if (experts > GINEX_MAX_EXPERTS) return false;
  w = {t.data_ptr(), (int32_t)experts, turned, width, out, stride, experts > 1 ? t.stride(0) : 0, type_of(t)};
  return true;
}

// A vector per layer, or none: false where it is neither.
bool vector_of(PyObject* o, int device, at::ScalarType type, int64_t rows, int64_t width, int64_t dims, const void*& v) {
  v = nullptr;
  if (o == Py_None) return true;
  at::Tensor t;
  if (!plain(o, device, t) || t.scalar_type() != type || t.dim() != dims || !t.is_contiguous()) return false;
  if (t.size(dims - 1) != width || (dims == 2 && t.size(0) != rows)) return false;
  v = t.data_ptr();
  return true;
}

bool routing_of(PyObject* offsets, PyObject* slot, PyObject* source, int device, ginex_routing_t& r) {
  at::Tensor o, s, f;
  if (!plain(offsets, device, o) || !plain(slot, device, s) || !plain(source, device, f)) return false;
  if (o.scalar_type() != at::kLong || s.scalar_type() != at::kInt || f.scalar_type() != at::kInt) return false;
  if (!o.is_contiguous() || !s.is_contiguous() || !f.is_contiguous()) return false;
  if (o.dim() != 1 || o.numel() < 2 || o.numel() - 1 > GINEX_MAX_EXPERTS || s.dim() != 2 || s.size(1) > INT32_MAX) return false;
  if (f.dim() != 1 || f.numel() != s.numel()) return false;
  r = {s.size(0), (int32_t)s.size(1), (int32_t)(o.numel() - 1), static_cast<int64_t*>(o.data_ptr()),
       static_cast<int32_t*>(s.data_ptr()), static_cast<int32_t*>(f.data_ptr())};
  return true;
}

at::Tensor space(size_t bytes, const at::Tensor& like) {
  return at::empty({(int64_t)bytes}, like.options().dtype(at::kByte));
}

void* stream_of(PyObject* o) { return PyLong_AsVoidPtr(o); }

bool number_of(PyObject* o, int64_t most, int64_t& v) {
  if (!PyLong_Check(o)) return false;
  int overflow = 0;
  v = PyLong_AsLongLongAndOverflow(o, &overflow);
  return overflow == 0 && v >= 0 && v <= most;
}

PyObject* answer(int32_t rc, std::initializer_list<at::Tensor> results) {
  PyObject* const tuple = PyTuple_New((Py_ssize_t)results.size() + 1);
  PyTuple_SET_ITEM(tuple, 0, PyLong_FromLong(rc));
  Py_ssize_t i = 1;
  for (const at::Tensor& t : results) PyTuple_SET_ITEM(tuple, i++, THPVariable_Wrap(t));
  return tuple;
}

// An allocation that fails is for the Python name to meet, as whatever else throws.
template <typename Go>
PyObject* guarded(Go go) {
  try {
    return go();
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// (device, stream, x, weight, bias, activation, residual, offsets, slot, source, by_slot)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 11) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const int device = (int)PyLong_AsLong(a[0]);
    at::Tensor x, weight, residual;
    ginex_rows_t from, to, and_;
    ginex_weights_t w;
    ginex_routing_t route;
    const void* bias;
    const bool routed = a[7] != Py_None, by_slot = a[10] == Py_True;
    int64_t activation;
    if (!number_of(a[5], INT32_MAX, activation)) Py_RETURN_NONE;
    if (!plain(a[2], device, x) || !plain(a[3], device, weight) || !rows_of(x, from)) Py_RETURN_NONE;
    if (!weights_of(weight, routed ? 3 : 2, x.scalar_type(), w)) Py_RETURN_NONE;
    if (routed && !routing_of(a[7], a[8], a[9], device, route)) Py_RETURN_NONE;
    if (!vector_of(a[4], device, x.scalar_type(), w.experts, w.out, routed ? 2 : 1, bias)) Py_RETURN_NONE;
    const int64_t slots = routed ? route.rows * route.top : from.rows;
    const bool has_residual = a[6] != Py_None;
    if (has_residual) {
      if (!plain(a[6], device, residual) || residual.scalar_type() != x.scalar_type() || !rows_of(residual, and_)) Py_RETURN_NONE;
      if (and_.rows != slots || and_.width != w.out) Py_RETURN_NONE;
    }
    if (!routed && by_slot) Py_RETURN_NONE;
    const at::Tensor y = at::empty({slots, w.out}, x.options());
    rows_of(y, to);
    void* const stream = stream_of(a[1]);
    const int32_t rc = unlocked([&] {
      return ginex_linear(&from, &w, bias, (int32_t)activation, has_residual ? &and_ : nullptr, routed ? &route : nullptr,
                          by_slot, &to, nullptr, stream);
    });
    return answer(rc, {y});
  });
}

// (device, stream, grad, offsets, slot, source)
PyObject* bias_gradient(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 6) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const int device = (int)PyLong_AsLong(a[0]);
    at::Tensor grad;
    ginex_rows_t from;
    ginex_routing_t route;
    const bool routed = a[3] != Py_None;
    if (!plain(a[2], device, grad) || !rows_of(grad, from)) Py_RETURN_NONE;
    if (routed && !routing_of(a[3], a[4], a[5], device, route)) Py_RETURN_NONE;
    const size_t need = ginex_bias_gradient_workspace_bytes(from.rows, routed ? route.experts : 1, from.width);
    if (need == 0) Py_RETURN_NONE;
    const at::TensorOptions f32 = grad.options().dtype(at::kFloat);
    const at::Tensor out = routed ? at::empty({route.experts, from.width}, f32) : at::empty({from.width}, f32);
    const at::Tensor ws = space(need, grad);
    void* const stream = stream_of(a[1]);
    const int32_t rc = unlocked([&] {
      return ginex_bias_gradient(&from, routed ? &route : nullptr, static_cast<float*>(out.data_ptr()), ws.data_ptr(), ws.numel(),
                                 stream);
    });
    return answer(rc, {out});
  });
}

// (device, stream, x, router, weight, bias, top, activation)
PyObject* expert_layer(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 8) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const int device = (int)PyLong_AsLong(a[0]);
    at::Tensor x, router, weight;
    ginex_rows_t from, by, to;
    ginex_weights_t w;
    const void* bias;
    if (!plain(a[2], device, x) || !plain(a[3], device, router) || !plain(a[4], device, weight)) Py_RETURN_NONE;
    if (!rows_of(x, from) || !rows_of(router, by) || router.scalar_type() != x.scalar_type()) Py_RETURN_NONE;
    if (!weights_of(weight, 3, x.scalar_type(), w)) Py_RETURN_NONE;
    if (!vector_of(a[5], device, x.scalar_type(), w.experts, w.out, 2, bias)) Py_RETURN_NONE;
    int64_t top, activation;
    if (!number_of(a[6], GINEX_MAX_FEW_TOP, top) || !number_of(a[7], INT32_MAX, activation)) Py_RETURN_NONE;
    const size_t need = ginex_expert_layer_workspace_bytes(from.rows, (int32_t)top, w.experts, w.width, w.out);
    if (need == 0) Py_RETURN_NONE;
    const at::Tensor y = at::empty({from.rows, w.out}, x.options()), ws = space(need, x);
    rows_of(y, to);
    void* const stream = stream_of(a[1]);
    const int32_t rc = unlocked([&] {
      return ginex_expert_layer(&from, &by, &w, bias, (int32_t)top, (int32_t)activation, &to, ws.data_ptr(), ws.numel(), stream);
    });
    return answer(rc, {y});
  });
}

// (device, stream, x, weight, bias, eps, stats)
PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 7) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const int device = (int)PyLong_AsLong(a[0]);
    at::Tensor x;
    ginex_rows_t from, to;
    const void *weight, *bias;
    if (!plain(a[2], device, x) || !rows_of(x, from) || !PyFloat_Check(a[5])) Py_RETURN_NONE;
    if (!vector_of(a[3], device, x.scalar_type(), 1, from.width, 1, weight)) Py_RETURN_NONE;
    if (!vector_of(a[4], device, x.scalar_type(), 1, from.width, 1, bias)) Py_RETURN_NONE;
    const at::Tensor y = at::empty({from.rows, from.width}, x.options());
    rows_of(y, to);
    const bool stats = a[6] == Py_True;
    const at::Tensor kept = stats ? at::empty({from.rows, 2}, x.options().dtype(at::kFloat)) : at::Tensor();
    const float eps = (float)PyFloat_AS_DOUBLE(a[5]);
    void* const stream = stream_of(a[1]);
    const int32_t rc = unlocked([&] {
      return ginex_layer_norm(&from, weight, bias, eps, &to, stats ? static_cast<float*>(kept.data_ptr()) : nullptr, stream);
    });
    return stats ? answer(rc, {y, kept}) : answer(rc, {y});
  });
}

// (device, stream, grad, x, stats, weight), with the vectors' gradients
PyObject* layer_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 6) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const int device = (int)PyLong_AsLong(a[0]);
    at::Tensor grad, x, stats;
    ginex_rows_t dy, from, to;
    const void* weight;
    if (!plain(a[2], device, grad) || !plain(a[3], device, x) || !plain(a[4], device, stats)) Py_RETURN_NONE;
    if (!rows_of(grad, dy) || !rows_of(x, from)) Py_RETURN_NONE;
    if (stats.scalar_type() != at::kFloat || stats.dim() != 2 || stats.size(0) != from.rows || stats.size(1) != 2 ||
        !stats.is_contiguous())
      Py_RETURN_NONE;
    if (!vector_of(a[5], device, x.scalar_type(), 1, from.width, 1, weight)) Py_RETURN_NONE;
    const size_t need = ginex_layer_norm_backward_workspace_bytes(from.rows, from.width);
    if (need == 0) Py_RETURN_NONE;
    const at::TensorOptions f32 = x.options().dtype(at::kFloat);
    const at::Tensor dx = at::empty({from.rows, from.width}, x.options()), dweight = at::empty({from.width}, f32);
    const at::Tensor dbias = at::empty({from.width}, f32), ws = space(need, x);
    rows_of(dx, to);
    void* const stream = stream_of(a[1]);
    const int32_t rc = unlocked([&] {
      return ginex_layer_norm_backward(&dy, &from, static_cast<float*>(stats.data_ptr()), weight, &to,
                                       static_cast<float*>(dweight.data_ptr()), static_cast<float*>(dbias.data_ptr()),
                                       ws.data_ptr(), ws.numel(), stream);
    });
    return answer(rc, {dx, dweight, dbias});
  });
}

bool ids_of(PyObject* o, int device, at::Tensor& ids) {
  return plain(o, device, ids) && ids.dim() == 1 && ids.is_contiguous() &&
         (ids.scalar_type() == at::kInt || ids.scalar_type() == at::kLong);
}

// (device, stream, table, ids, scale)
PyObject* lookup(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 5) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const int device = (int)PyLong_AsLong(a[0]);
    at::Tensor table, ids;
    ginex_rows_t from, to;
    if (!plain(a[2], device, table) || !ids_of(a[3], device, ids) || !rows_of(table, from) || !PyFloat_Check(a[4])) Py_RETURN_NONE;
    const at::Tensor out = at::empty({ids.numel(), from.width}, table.options());
    rows_of(out, to);
    const float scale = (float)PyFloat_AS_DOUBLE(a[4]);
    void* const stream = stream_of(a[1]);
    const int32_t rc = unlocked([&] {
      return ginex_lookup(&from, ids.data_ptr(), ids.scalar_type() == at::kLong, scale, &to, stream);
    });
    return answer(rc, {out});
  });
}

// (device, stream, grad, ids, rows, scale)
PyObject* lookup_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 6) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const int device = (int)PyLong_AsLong(a[0]);
    at::Tensor grad, ids;
    ginex_rows_t dy, to;
    int64_t rows;
    if (!plain(a[2], device, grad) || !ids_of(a[3], device, ids) || !rows_of(grad, dy) || !PyFloat_Check(a[5])) Py_RETURN_NONE;
    if (!number_of(a[4], INT64_MAX, rows) || ids.numel() != dy.rows) Py_RETURN_NONE;
    const size_t need = ginex_lookup_backward_workspace_bytes(dy.rows, rows, dy.width);
    if (need == 0) Py_RETURN_NONE;
    const at::Tensor out = at::empty({rows, dy.width}, grad.options()), ws = space(need, grad);
    rows_of(out, to);
    const float scale = (float)PyFloat_AS_DOUBLE(a[5]);
    void* const stream = stream_of(a[1]);
    const int32_t rc = unlocked([&] {
      return ginex_lookup_backward(&dy, ids.data_ptr(), ids.scalar_type() == at::kLong, scale, &to, ws.data_ptr(), ws.numel(),
                                   stream);
    });
    return answer(rc, {out});
  });
}

#define QUICK(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {QUICK(linear), QUICK(bias_gradient), QUICK(expert_layer), QUICK(layer_norm), QUICK(layer_norm_backward),
                         QUICK(lookup), QUICK(lookup_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_quick", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__quick() { return PyModule_Create(&module); }
