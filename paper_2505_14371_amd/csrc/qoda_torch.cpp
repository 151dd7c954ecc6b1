// The torch-facing code's look at its tensors, in native code.  The loop's K x L gradients: every tensor is looked at in every round, and in a
// small model that was most of the host's time (four lists of 17 tensors: 20 us in Python, under 2 here).  The operators' arguments: a call
// on small tensors took the host 9 to 13 us in Python, and the device 5.  A module of the interpreter, not part of libqoda's C ABI.
#include <ATen/ops/empty.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/qoda_matrices.h"

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

PyObject *used(PyObject *addresses, void *to, size_t bytes, const char *said) {
  void *p[32];
  const Py_ssize_t n = (Py_ssize_t)(bytes / sizeof(void *));
  if (!PyTuple_CheckExact(addresses) || PyTuple_GET_SIZE(addresses) != n) {
    PyErr_SetString(PyExc_TypeError, said);
    return nullptr;
  }
  for (Py_ssize_t i = 0; i < n; ++i) {
    p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(addresses, i));
    if (PyErr_Occurred()) return nullptr;
  }
  memcpy(to, p, bytes);
  Py_RETURN_NONE;
}

// use(addresses): the calls above, in their order.
PyObject *use(PyObject *, PyObject *addresses) { return used(addresses, &calls, sizeof calls, "use(addresses)"); }

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

// ---- include/qoda_matrices.h

struct MatrixCalls {
  decltype(&qoda_mx_quantize) quantize;
  decltype(&qoda_mx_values) values;
  decltype(&qoda_mx_linear_workspace_bytes) linear_bytes;
  decltype(&qoda_mx_linear) linear;
  decltype(&qoda_mx_linear_input_grad_workspace_bytes) input_grad_bytes;
  decltype(&qoda_mx_linear_input_grad) input_grad;
  decltype(&qoda_mx_linear_weight_grad_workspace_bytes) weight_grad_bytes;
  decltype(&qoda_mx_linear_weight_grad) weight_grad;
  decltype(&qoda_orthogonalize_workspace_bytes) orthogonalize_bytes;
  decltype(&qoda_orthogonalize) orthogonalize;
} matrix_calls;

// use_matrices(addresses): the calls above, in their order.
PyObject *use_matrices(PyObject *, PyObject *addresses) { return used(addresses, &matrix_calls, sizeof matrix_calls, "use_matrices(addresses)"); }

// A microscaled matrix, as (codes, scales, rows, columns): the caller's class has looked at their shapes; scales None: they lie behind the codes.
struct Mx {
  const at::Tensor &codes;
  int64_t rows, cols;
  void *scales;
  Mx(PyObject *o, int64_t device) : codes(tensor(part(o, 0))), rows(number<int64_t>(part(o, 2))), cols(number<int64_t>(part(o, 3))) {
    if (!codes.is_cuda() || codes.get_device() != device) throw Unknown();
    if (part(o, 1) == Py_None) {
      scales = static_cast<char *>(codes.data_ptr()) + code_bytes(rows, cols);
    } else {
      const at::Tensor &t = tensor(part(o, 1));
      if (!t.is_cuda() || t.get_device() != device) throw Unknown();
      scales = t.data_ptr();
    }
  }
  static int64_t code_bytes(int64_t rows, int64_t cols) { return rows * ((cols + 255) / 256 * 128); }
  static PyObject *part(PyObject *o, Py_ssize_t i) {
    if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 4) throw Unknown();
    return PyTuple_GET_ITEM(o, i);
  }
  qoda_mx as_is() const { return {codes.data_ptr(), scales}; }
};

at::Tensor bytes_of(const at::Tensor &like, at::IntArrayRef sizes) { return at::empty(sizes, like.options().dtype(at::kByte)); }

// (device, stream, x, transposed, stochastic, seed, offset): (codes and scales, None, rows, columns)
PyObject *microscale(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  return answered(args, nargs, 7, [&](int64_t device, void *stream) {
    if (!matrix_calls.quantize) throw Unknown();
    not_followed({args[2]});
    const First x(args[2], device, 1);
    const bool transposed = truth(args[3]);
    const int64_t rows = transposed ? x.cols : x.rows, cols = transposed ? x.rows : x.cols, steps = (cols + 255) / 256;
    if (rows > QODA_MAX_SIDE || cols > QODA_MAX_SIDE) throw Unknown();
    const int64_t codes = Mx::code_bytes(rows, cols), scales = (rows + 63) / 64 * 512 * steps;
    const at::Tensor q = bytes_of(x.t, {codes + scales});
    const qoda_mx_quantize_args a = {x.dtype, transposed, truth(args[4]), x.rows, x.cols, matrix(args[2], x, x.rows, x.cols),
                                     {q.data_ptr(), static_cast<char *>(q.data_ptr()) + codes}, number<uint64_t>(args[5]), number<uint64_t>(args[6])};
    const int rc = matrix_calls.quantize(&a, stream);
    if (rc != QODA_OK) return PyLong_FromLong(rc);
    return Py_BuildValue("(NOLL)", THPVariable_Wrap(q), Py_None, (long long)rows, (long long)cols);
  });
}

// The rows of a product's first operand: plain, or microscaled with a type for what goes with them.
struct Rows {
  const at::Tensor *t;      // whose device and, plain, type the others have
  at::ScalarType type;
  int32_t dtype;
  int64_t rows, cols;
  qoda_matrix plain = {nullptr, 0};
  qoda_mx mx = {nullptr, nullptr};
  c10::SmallVector<int64_t, 6> front;
  Rows(PyObject *o, PyObject *bf16, int64_t device) {
    if (PyTuple_CheckExact(o)) {
      const Mx q(o, device);
      t = &q.codes, rows = q.rows, cols = q.cols, mx = q.as_is();
      dtype = truth(bf16) ? QODA_BF16 : QODA_F32;
      type = dtype == QODA_BF16 ? at::kBFloat16 : at::kFloat;
      front = {rows};
    } else {
      if (bf16 != Py_None) throw Unknown();
      const First x(o, device, 1);
      t = &x.t, rows = x.rows, cols = x.cols, dtype = x.dtype, type = x.t.scalar_type();
      plain = matrix(o, x, rows, cols);
      front.assign(x.t.sizes().begin(), x.t.sizes().end() - 1);
    }
  }
  at::Tensor output(int64_t columns) const {
    c10::SmallVector<int64_t, 6> sizes = front;
    sizes.push_back(columns);
    return at::empty(sizes, t->options().dtype(type));
  }
  qoda_matrix beside(PyObject *o, const First &like, int64_t columns) const { return matrix(o, like, rows, columns); }
};

// First of a tensor that this code has made: its type and device are what other arguments are compared with.
First made(const at::Tensor &t, PyObject *&holder, int64_t device) {
  holder = THPVariable_Wrap(t);
  return First(holder, device, 1);
}
struct Held {   // a reference that goes with the scope
  PyObject *o = nullptr;
  ~Held() { Py_XDECREF(o); }
};

// The call with its workspace on the device of `like`: 0, or the library's error code.
template <class Args, class Bytes, class Call>
int with_scratch(const at::Tensor &like, const Args &a, Bytes bytes, Call call, void *stream) {
  const int64_t need = bytes(&a);
  if (need < 0) return (int)need;
  at::Tensor scratch;
  if (need > 0) scratch = bytes_of(like, {need});
  return call(&a, need > 0 ? scratch.data_ptr() : nullptr, (size_t)need, stream);
}

// (device, stream, x, weight, bias, residual, activation, p, seed, offset, keep_pre, bf16); bf16: of the outputs, None where x is plain
PyObject *mx_linear(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  return answered(args, nargs, 12, [&](int64_t device, void *stream) {
    if (!matrix_calls.linear) throw Unknown();
    if (!PyTuple_CheckExact(args[2])) not_followed({args[2]});
    not_followed({args[4], args[5]});
    const Rows x(args[2], args[11], device);
    const Mx w(args[3], device);
    if (w.cols != x.cols) throw Unknown();
    const at::Tensor y = x.output(w.rows);
    Held held;
    const First like = made(y, held.o, device);
    qoda_mx_linear_args a = {x.dtype, (int32_t)number<int64_t>(args[6]), x.rows, x.cols, w.rows, x.plain, x.mx, w.as_is(), x.beside(args[5], like, w.rows),
                             {y.data_ptr(), w.rows}, {}, vector(args[4], like, w.rows), number<double>(args[7]), number<uint64_t>(args[8]), number<uint64_t>(args[9])};
    if (!truth(args[10])) return outcome(with_scratch(y, a, matrix_calls.linear_bytes, matrix_calls.linear, stream), {y});
    const at::Tensor pre = x.output(w.rows);
    a.pre = {pre.data_ptr(), w.rows};
    return outcome(with_scratch(y, a, matrix_calls.linear_bytes, matrix_calls.linear, stream), {y, pre});
  });
}

// (device, stream, dz, weight_t, pre, activation, p, seed, offset, residual, bf16)
PyObject *mx_linear_input_grad(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  return answered(args, nargs, 11, [&](int64_t device, void *stream) {
    if (!matrix_calls.input_grad) throw Unknown();
    const Rows dz(args[2], args[10], device);
    const Mx wt(args[3], device);
    if (wt.cols != dz.cols) throw Unknown();
    const at::Tensor dx = dz.output(wt.rows);
    Held held;
    const First like = made(dx, held.o, device);
    const qoda_mx_linear_input_grad_args a = {dz.dtype, (int32_t)number<int64_t>(args[5]), dz.rows, wt.rows, dz.cols, dz.plain, dz.mx, wt.as_is(), dz.beside(args[4], like, wt.rows),
                                              dz.beside(args[9], like, wt.rows), {dx.data_ptr(), wt.rows}, number<double>(args[6]), number<uint64_t>(args[7]),
                                              number<uint64_t>(args[8])};
    return outcome(with_scratch(dx, a, matrix_calls.input_grad_bytes, matrix_calls.input_grad, stream), {dx});
  });
}

// (device, stream, dz_t, x_t, dweight, dbias, accumulate), with both outputs given (dbias may be None); answers with True
PyObject *mx_linear_weight_grad(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  return answered(args, nargs, 7, [&](int64_t device, void *stream) -> PyObject * {
    if (!matrix_calls.weight_grad) throw Unknown();
    const Mx dzt(args[2], device), xt(args[3], device);
    if (dzt.cols != xt.cols || args[4] == Py_None) throw Unknown();
    const First dw(args[4], device, 2);
    if (dw.dtype != QODA_F32) throw Unknown();
    const qoda_mx_linear_weight_grad_args a = {truth(args[6]), dzt.cols, xt.rows, dzt.rows, dzt.as_is(), xt.as_is(), matrix(args[4], dw, dzt.rows, xt.rows), vector(args[5], dw, dzt.rows)};
    const int rc = with_scratch(dzt.codes, a, matrix_calls.weight_grad_bytes, matrix_calls.weight_grad, stream);
    if (rc != QODA_OK) return PyLong_FromLong(rc);
    Py_RETURN_TRUE;
  });
}

// (device, stream, q, bf16)
PyObject *mx_values(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  return answered(args, nargs, 4, [&](int64_t device, void *stream) {
    if (!matrix_calls.values) throw Unknown();
    const Mx q(args[2], device);
    const bool wide = !truth(args[3]);
    const at::Tensor y = at::empty({q.rows, q.cols}, q.codes.options().dtype(wide ? at::kFloat : at::kBFloat16));
    const qoda_mx_values_args a = {wide ? QODA_F32 : QODA_BF16, q.rows, q.cols, q.as_is(), {y.data_ptr(), q.cols}};
    return outcome(matrix_calls.values(&a, stream), {y});
  });
}

// (device, stream, g, steps, a, b, c, eps, out); out: None makes it
PyObject *orthogonalize(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  return answered(args, nargs, 9, [&](int64_t device, void *stream) {
    if (!matrix_calls.orthogonalize) throw Unknown();
    not_followed({args[2], args[8]});
    const First g(args[2], device, 2);
    const int64_t rows = g.t.size(g.t.dim() - 2), n = rows > 0 ? g.rows / rows : 0;
    const auto places = [&](const at::Tensor &t) -> qoda_matrices {
      if (t.is_contiguous()) return {t.data_ptr(), rows * g.cols, g.cols};
      if (t.dim() > 3 || (g.cols > 1 && t.stride(t.dim() - 1) != 1)) throw Unknown();
      return {t.data_ptr(), t.dim() == 3 ? t.stride(0) : 0, t.stride(t.dim() - 2)};
    };
    const at::Tensor x = args[8] == Py_None ? rows_of(g, g.cols) : tensor(args[8]);
    if (rows == 0 || !x.is_cuda() || x.get_device() != device || x.scalar_type() != g.t.scalar_type() || x.sizes() != g.t.sizes()) throw Unknown();
    const int64_t steps = number<int64_t>(args[3]);
    if (steps > INT32_MAX || steps < INT32_MIN) throw Unknown();
    const qoda_orthogonalize_args a = {g.dtype, (int32_t)steps, n, rows, g.cols, places(g.t), places(x), number<double>(args[4]), number<double>(args[5]), number<double>(args[6]),
                                       number<double>(args[7])};
    const int rc = with_scratch(g.t, a, matrix_calls.orthogonalize_bytes, matrix_calls.orthogonalize, stream);
    if (rc == QODA_OK && args[8] != Py_None) {
      Py_INCREF(args[8]);
      return args[8];
    }
    return outcome(rc, {x});
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
                         {"use_matrices", use_matrices, METH_O, nullptr},
                         {"microscale", fast(microscale), METH_FASTCALL, nullptr},
                         {"mx_values", fast(mx_values), METH_FASTCALL, nullptr},
                         {"mx_linear", fast(mx_linear), METH_FASTCALL, nullptr},
                         {"mx_linear_input_grad", fast(mx_linear_input_grad), METH_FASTCALL, nullptr},
                         {"mx_linear_weight_grad", fast(mx_linear_weight_grad), METH_FASTCALL, nullptr},
                         {"orthogonalize", fast(orthogonalize), METH_FASTCALL, nullptr},
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
