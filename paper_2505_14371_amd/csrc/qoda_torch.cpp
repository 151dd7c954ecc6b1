// The torch-facing code's look at its tensors, in native code.  The loop's K x L gradients: every tensor is looked at in every round, and in a
// small model that was most of the host's time (four lists of 17 tensors: 20 us in Python, under 2 here).  The operators' arguments: a call
// on small tensors took the host 9 to 13 us in Python, and the device 5.  A module of the interpreter, not part of libqoda's C ABI.
#include <ATen/ops/empty.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/qoda_operators.h"

#include <cstdint>
#include <cstring>
#include <initializer_list>
#include <type_traits>

namespace {

// A plain tensor or parameter; anything else (a subclass may answer for itself) is left to the caller's own look.
const at::Tensor *plain_tensor(PyObject *o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

// gather(node_grads, params, nodes, out): whether node_grads is a list or tuple of `nodes` lists or tuples of contiguous fp32 CUDA tensors with the
// parameters' numbers of elements; if so, their addresses are stored at out, node by node.  False also where that cannot be told here.
PyObject *gather(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  if (nargs != 4) {
    PyErr_SetString(PyExc_TypeError, "gather(node_grads, params, nodes, out)");
    return nullptr;
  }
  PyObject *lists = args[0], *params = args[1];
  const Py_ssize_t nodes = PyLong_AsSsize_t(args[2]);
  uint64_t *out = static_cast<uint64_t *>(PyLong_AsVoidPtr(args[3]));
  if (PyErr_Occurred()) return nullptr;
  const auto plain = [](PyObject *o) { return PyList_CheckExact(o) || PyTuple_CheckExact(o); };
  if (!plain(lists) || !plain(params) || PySequence_Fast_GET_SIZE(lists) != nodes) Py_RETURN_FALSE;
  const Py_ssize_t L = PySequence_Fast_GET_SIZE(params);
  try {
    for (Py_ssize_t k = 0; k < nodes; ++k) {
      PyObject *g = PySequence_Fast_GET_ITEM(lists, k);
      if (!plain(g) || PySequence_Fast_GET_SIZE(g) != L) Py_RETURN_FALSE;
      for (Py_ssize_t l = 0; l < L; ++l) {
        const at::Tensor *t = plain_tensor(PySequence_Fast_GET_ITEM(g, l)), *p = plain_tensor(PySequence_Fast_GET_ITEM(params, l));
        if (!t || !p || !t->is_cuda() || t->scalar_type() != at::kFloat || !t->is_contiguous() || t->numel() != p->numel()) Py_RETURN_FALSE;
        out[k * L + l] = reinterpret_cast<uint64_t>(t->data_ptr());
      }
    }
  } catch (...) {   // a tensor without memory of its own, say: the caller's look reports it
    Py_RETURN_FALSE;
  }
  Py_RETURN_TRUE;
}

// ---- operators.  Each function takes a call's arguments, with the activation's number and the device and stream that are current in front,
// and answers with the outputs, or with the library's error code, or with None where the arguments are not what it knows how to pass on: the caller's own
// code looks at them then, and says what is wrong.

struct Calls {   // of the library that the caller has loaded
  decltype(&qoda_linear_workspace_bytes) linear_bytes;
  decltype(&qoda_linear) linear;
  decltype(&qoda_linear_input_grad_workspace_bytes) input_grad_bytes;
  decltype(&qoda_linear_input_grad) input_grad;
  decltype(&qoda_linear_weight_grad_workspace_bytes) weight_grad_bytes;
  decltype(&qoda_linear_weight_grad) weight_grad;
  decltype(&qoda_dropout) dropout;
  decltype(&qoda_dropout_grad) dropout_grad;
  decltype(&qoda_group_norm_workspace_bytes) norm_bytes;
  decltype(&qoda_group_norm) norm;
  decltype(&qoda_group_norm_grad_workspace_bytes) norm_grad_bytes;
  decltype(&qoda_group_norm_grad) norm_grad;
} calls;

// use(addresses): the calls above, in their order.
PyObject *use(PyObject *, PyObject *addresses) {
  constexpr Py_ssize_t n = sizeof calls / sizeof(void *);
  if (!PyTuple_CheckExact(addresses) || PyTuple_GET_SIZE(addresses) != n) {
    PyErr_SetString(PyExc_TypeError, "use(addresses)");
    return nullptr;
  }
  void *p[n];
  for (Py_ssize_t i = 0; i < n; ++i) {
    p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(addresses, i));
    if (PyErr_Occurred()) return nullptr;
  }
  memcpy(&calls, p, sizeof p);
  Py_RETURN_NONE;
}

struct Unknown {};   // thrown inside a function whose arguments are not plain

const at::Tensor &tensor(PyObject *o) {
  const at::Tensor *t = plain_tensor(o);
  if (!t || !t->defined()) throw Unknown();
  return *t;
}

// Tensors that torch is to differentiate by: for the caller's own code, which answers with what says that nothing is recorded.
void not_followed(std::initializer_list<PyObject *> inputs) {
  const bool recording = c10::GradMode::is_enabled();
  for (PyObject *o : inputs) {
    if (o == Py_None) continue;
    const at::Tensor &t = tensor(o);
    if ((recording && t.requires_grad()) || t._fw_grad(0).defined()) throw Unknown();
  }
}

// A call's first tensor: its rows and columns, type and device are the call's.
struct First {
  const at::Tensor &t;
  int64_t rows = 1, cols;
  int32_t dtype;
  First(PyObject *o, int64_t device, int64_t least_dims) : t(tensor(o)) {
    if (!t.is_cuda() || t.get_device() != device || t.dim() < least_dims) throw Unknown();
    if (t.scalar_type() == at::kFloat) dtype = QODA_F32;
    else if (t.scalar_type() == at::kBFloat16) dtype = QODA_BF16;
    else throw Unknown();
    for (int64_t d = 0; d + 1 < t.dim(); ++d) rows *= t.size(d);
    cols = t.size(t.dim() - 1);
  }
};

qoda_matrix matrix(PyObject *o, const First &like, int64_t rows, int64_t cols, bool fp32 = false) {
  if (o == Py_None) return {nullptr, 0};
  const at::Tensor &t = tensor(o);
  if (!t.is_cuda() || t.get_device() != like.t.get_device() || t.scalar_type() != (fp32 ? at::kFloat : like.t.scalar_type())) throw Unknown();
  if (t.dim() == 2) {
    if (t.size(0) != rows || t.size(1) != cols || (cols > 1 && t.stride(1) != 1)) throw Unknown();
    return {t.data_ptr(), t.stride(0)};
  }
  if (t.dim() == 0 || !t.is_contiguous() || t.size(t.dim() - 1) != cols || t.numel() != rows * cols) throw Unknown();
  return {t.data_ptr(), cols};
}

float *vector(PyObject *o, const First &like, int64_t n) {
  if (o == Py_None) return nullptr;
  const at::Tensor &t = tensor(o);
  if (!t.is_cuda() || t.get_device() != like.t.get_device() || t.scalar_type() != at::kFloat || t.numel() != n || !t.is_contiguous()) throw Unknown();
  return static_cast<float *>(t.data_ptr());
}

qoda_channels_last values(PyObject *o, const First &like) {
  if (o == Py_None) return {nullptr, 0, 0};
  const at::Tensor &t = tensor(o);
  if (!t.is_cuda() || t.get_device() != like.t.get_device() || t.scalar_type() != like.t.scalar_type() || t.sizes() != like.t.sizes()) throw Unknown();
  if (t.is_contiguous()) return {t.data_ptr(), t.size(0) > 0 ? t.numel() / t.size(0) : 0, like.cols};
  if (t.dim() != 3 || (like.cols > 1 && t.stride(2) != 1)) throw Unknown();
  return {t.data_ptr(), t.stride(0), t.stride(1)};
}

template <class T>
T number(PyObject *o) {
  T v;
  if constexpr (std::is_same_v<T, double>) v = PyFloat_AsDouble(o);
  else if constexpr (std::is_same_v<T, uint64_t>) v = PyLong_AsUnsignedLongLong(o);
  else v = PyLong_AsLongLong(o);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    throw Unknown();
  }
  return v;
}
bool truth(PyObject *o) {
  if (o != Py_True && o != Py_False) throw Unknown();
  return o == Py_True;
}

at::Tensor output(const First &like, at::IntArrayRef sizes, at::ScalarType type) { return at::empty(sizes, like.t.options().dtype(type)); }
at::Tensor rows_of(const First &like, int64_t cols) {
  c10::SmallVector<int64_t, 6> sizes(like.t.sizes().begin(), like.t.sizes().end());
  sizes.back() = cols;
  return output(like, sizes, like.t.scalar_type());
}

// The call with its workspace: 0, or the library's error code.
template <class Args, class Bytes, class Call>
int with_workspace(const First &like, const Args &a, Bytes bytes, Call call, void *stream) {
  const int64_t need = bytes(&a);
  if (need < 0) return (int)need;
  at::Tensor scratch;
  if (need > 0) scratch = output(like, {need}, at::kByte);
  return call(&a, need > 0 ? scratch.data_ptr() : nullptr, (size_t)need, stream);
}

// Runs body(device, stream) -> a new reference, for a call of `wanted` arguments, device and stream the first two.
template <class F>
PyObject *answered(PyObject *const *args, Py_ssize_t nargs, Py_ssize_t wanted, F &&body) {
  if (nargs != wanted || !calls.linear) {
    PyErr_SetString(PyExc_TypeError, "another number of arguments, or the library's calls are not known");
    return nullptr;
  }
  try {
    return body(number<int64_t>(args[0]), reinterpret_cast<void *>(number<uint64_t>(args[1])));
  } catch (const Unknown &) {
  } catch (...) {   // no memory, say: the caller's own call reports it
  }
  Py_RETURN_NONE;
}
PyObject *outcome(int rc, std::initializer_list<at::Tensor> outputs) {
  if (rc != QODA_OK) return PyLong_FromLong(rc);
  if (outputs.size() == 1) return THPVariable_Wrap(*outputs.begin());
  PyObject *r = PyTuple_New((Py_ssize_t)outputs.size());
  Py_ssize_t i = 0;
  for (const at::Tensor &t : outputs) PyTuple_SET_ITEM(r, i++, THPVariable_Wrap(t));
  return r;
}

// (device, stream, x, weight, bias, residual, activation, p, seed, offset, keep_pre)
PyObject *linear(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  return answered(args, nargs, 11, [&](int64_t device, void *stream) {
    not_followed({args[2], args[3], args[4], args[5]});
    const First x(args[2], device, 1);
    const at::Tensor &w = tensor(args[3]);
    if (w.dim() != 2) throw Unknown();
    const int64_t out = w.size(0);
    qoda_linear_args a = {x.dtype, (int32_t)number<int64_t>(args[6]), x.rows, x.cols, out, matrix(args[2], x, x.rows, x.cols), matrix(args[3], x, out, x.cols),
                          matrix(args[5], x, x.rows, out), {}, {}, vector(args[4], x, out), number<double>(args[7]), number<uint64_t>(args[8]), number<uint64_t>(args[9])};
    const at::Tensor y = rows_of(x, out);
    a.y = {y.data_ptr(), out};
    if (!truth(args[10])) return outcome(with_workspace(x, a, calls.linear_bytes, calls.linear, stream), {y});
    const at::Tensor pre = rows_of(x, out);
    a.pre = {pre.data_ptr(), out};
    return outcome(with_workspace(x, a, calls.linear_bytes, calls.linear, stream), {y, pre});
  });
}

// (device, stream, dz, weight, pre, activation, p, seed, offset, residual)
PyObject *linear_input_grad(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  return answered(args, nargs, 10, [&](int64_t device, void *stream) {
    const First dz(args[2], device, 1);
    const at::Tensor &w = tensor(args[3]);
    if (w.dim() != 2) throw Unknown();
    const int64_t in = w.size(1);
    qoda_linear_input_grad_args a = {dz.dtype, (int32_t)number<int64_t>(args[5]), dz.rows, in, dz.cols, matrix(args[2], dz, dz.rows, dz.cols),
                                     matrix(args[3], dz, dz.cols, in), matrix(args[4], dz, dz.rows, in), matrix(args[9], dz, dz.rows, in), {},
                                     number<double>(args[6]), number<uint64_t>(args[7]), number<uint64_t>(args[8])};
    const at::Tensor dx = rows_of(dz, in);
    a.dx = {dx.data_ptr(), in};
    return outcome(with_workspace(dz, a, calls.input_grad_bytes, calls.input_grad, stream), {dx});
  });
}

// (device, stream, dz, x, dweight, dbias, accumulate), with both outputs given; answers with True
PyObject *linear_weight_grad(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  return answered(args, nargs, 7, [&](int64_t device, void *stream) -> PyObject * {
    const First dz(args[2], device, 1);
    const at::Tensor &x = tensor(args[3]);
    if (x.dim() == 0 || args[4] == Py_None) throw Unknown();
    const int64_t in = x.size(x.dim() - 1);
    const qoda_linear_weight_grad_args a = {dz.dtype, truth(args[6]), dz.rows, in, dz.cols, matrix(args[2], dz, dz.rows, dz.cols), matrix(args[3], dz, dz.rows, in),
                                            matrix(args[4], dz, dz.cols, in, true), vector(args[5], dz, dz.cols)};
    const int rc = with_workspace(dz, a, calls.weight_grad_bytes, calls.weight_grad, stream);
    if (rc != QODA_OK) return PyLong_FromLong(rc);
    Py_RETURN_TRUE;
  });
}

// (device, stream, x, extra, activation, p, seed, offset, gradient)
PyObject *entries(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  return answered(args, nargs, 9, [&](int64_t device, void *stream) {
    if (!truth(args[8])) not_followed({args[2], args[3]});
    const First x(args[2], device, 1);
    qoda_dropout_args a = {x.dtype, (int32_t)number<int64_t>(args[4]), x.rows, x.cols, matrix(args[2], x, x.rows, x.cols), matrix(args[3], x, x.rows, x.cols), {},
                           number<double>(args[5]), number<uint64_t>(args[6]), number<uint64_t>(args[7])};
    const at::Tensor y = rows_of(x, x.cols);
    a.y = {y.data_ptr(), x.cols};
    return outcome((truth(args[8]) ? calls.dropout_grad : calls.dropout)(&a, stream), {y});
  });
}

// (device, stream, x, groups, weight, bias, eps, activation)
PyObject *group_norm(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  return answered(args, nargs, 8, [&](int64_t device, void *stream) {
    not_followed({args[2], args[4], args[5]});
    const First x(args[2], device, 2);
    const int64_t n = x.t.size(0), groups = number<int64_t>(args[3]);
    if (groups < 1 || x.t.numel() == 0) throw Unknown();
    const int64_t positions = x.rows / n;
    const at::Tensor y = rows_of(x, x.cols), mean = output(x, {n, groups}, at::kFloat), rstd = output(x, {n, groups}, at::kFloat);
    const qoda_group_norm_args a = {x.dtype, (int32_t)number<int64_t>(args[7]), n, positions, x.cols, groups, values(args[2], x), {y.data_ptr(), positions * x.cols, x.cols},
                                    vector(args[4], x, x.cols), vector(args[5], x, x.cols), static_cast<float *>(mean.data_ptr()), static_cast<float *>(rstd.data_ptr()),
                                    number<double>(args[6])};
    return outcome(with_workspace(x, a, calls.norm_bytes, calls.norm, stream), {y, mean, rstd});
  });
}

// (device, stream, dy, x, mean, rstd, groups, weight, bias, activation, residual, dweight, dbias, accumulate); dweight, dbias: None makes them
PyObject *group_norm_grad(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  return answered(args, nargs, 14, [&](int64_t device, void *stream) {
    const First x(args[3], device, 2);
    const int64_t n = x.t.size(0), groups = number<int64_t>(args[6]), c = x.cols;
    if (groups < 1 || n == 0) throw Unknown();
    const int64_t positions = x.rows / n;
    const at::Tensor dx = rows_of(x, c), dw = args[11] == Py_None ? output(x, {c}, at::kFloat) : tensor(args[11]),
                     db = args[12] == Py_None ? output(x, {c}, at::kFloat) : tensor(args[12]);
    qoda_group_norm_grad_args a = {x.dtype, (int32_t)number<int64_t>(args[9]), n, positions, c, groups, values(args[2], x), values(args[3], x), values(args[10], x),
                                   {dx.data_ptr(), positions * c, c}, vector(args[7], x, c), vector(args[8], x, c), vector(args[4], x, n * groups), vector(args[5], x, n * groups),
                                   args[11] == Py_None ? static_cast<float *>(dw.data_ptr()) : vector(args[11], x, c),
                                   args[12] == Py_None ? static_cast<float *>(db.data_ptr()) : vector(args[12], x, c), truth(args[13])};
    return outcome(with_workspace(x, a, calls.norm_grad_bytes, calls.norm_grad, stream), {dx, dw, db});
  });
}

PyCFunction fast(PyObject *(*f)(PyObject *, PyObject *const *, Py_ssize_t)) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {{"gather", fast(gather), METH_FASTCALL, nullptr},
                         {"use", use, METH_O, nullptr},
                         {"linear", fast(linear), METH_FASTCALL, nullptr},
                         {"linear_input_grad", fast(linear_input_grad), METH_FASTCALL, nullptr},
                         {"linear_weight_grad", fast(linear_weight_grad), METH_FASTCALL, nullptr},
                         {"entries", fast(entries), METH_FASTCALL, nullptr},
                         {"group_norm", fast(group_norm), METH_FASTCALL, nullptr},
                         {"group_norm_grad", fast(group_norm_grad), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_qoda_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__qoda_torch() {
  PyObject *m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_for", QODA_BUILT_FOR) != 0) {   // the caller compares it with what is running
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
