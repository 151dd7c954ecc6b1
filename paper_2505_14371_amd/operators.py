"""Thin binding over the operators of include/qoda_operators.h: the matrix product with its epilogue, dropout, group normalisation, and
their gradients, on torch tensors.

Argument marshalling only, as in ``qoda``: every operator runs in the library's HIP kernels, and there is no CPU fallback.  Outputs and
scratch memory come from torch's allocator, on the stream that the call runs on (``stream``: a torch stream or a handle; None: the
current one).

    y, z = linear(x, w, b, activation="gelu", p=0.1, seed=s, offset=o, keep_pre=True)     # y = drop(gelu(x w^T + b)), z before gelu
    y2 = linear(y, w2, b2, residual=x, p=0.1, seed=s, offset=o + 1)                       # x + drop(y w2^T + b2)
    dz2 = dropout_grad(dy2, p=0.1, seed=s, offset=o + 1)
    dz = linear_input_grad(dz2, w2, pre=z, activation="gelu", p=0.1, seed=s, offset=o)    # back through w2, the dropout and gelu
    linear_weight_grad(dz2, y, dweight=g_w2, dbias=g_b2)                                  # fp32, into the vector that is quantized

Matrices are tensors of fp32 or bfloat16 whose last dimension is adjacent; the dimensions before it are rows.  Biases, scales,
statistics and gradients of parameters are fp32.  ``activation``: "none", "relu", "leaky_relu" (slope 0.2), "gelu" or "silu".
Dropout keeps entry (r, c) by a draw that (seed, offset, r, c) fixes, so that a gradient call with the same p, seed and offset
has the forward call's mask; two calls whose masks are to differ have different offsets.

Each operator has its gradient as a call of its own, and nothing is recorded for torch's differentiation.  Outputs of ``linear``, ``dropout``
and ``group_norm`` on tensors that require a gradient, outside ``torch.no_grad()``, require one too, and raise where it is asked for; tangents
are refused.  What the gradient calls return is plain.
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional, Tuple

import torch

from . import build, qoda

ACTIVATIONS = {"none": 0, "relu": 1, "leaky_relu": 2, "gelu": 3, "silu": 4}
DTYPES = {torch.float32: 0, torch.bfloat16: 1}

# the argument structures of the header, packed as C lays them out
_LINEAR = struct.Struct("@2i3q" + "Pq" * 5 + "PdQQ")
_INPUT_GRAD = struct.Struct("@2i3q" + "Pq" * 5 + "dQQ")
_WEIGHT_GRAD = struct.Struct("@2i3q" + "Pq" * 3 + "P")
_DROPOUT = struct.Struct("@2i2q" + "Pq" * 3 + "dQQ")
_NORM = struct.Struct("@2i4q" + "Pqq" * 2 + "4Pd")
_NORM_GRAD = struct.Struct("@2i4q" + "Pqq" * 4 + "6Pi0q")

_lib = None
_native = None          # the native look at the arguments, once the library is loaded
_ready = False          # whether torch has been seen to have a device
# the current device and its current stream's handle, without a Stream object; not public functions of torch
_get_device, _get_stream = (getattr(torch._C, n, None) for n in ("_cuda_getDevice", "_cuda_getCurrentRawStream"))


def _find_native(L):
    """csrc/qoda_torch.cpp's functions, if they are there and were built for this torch, given the library's calls."""
    try:
        from . import _qoda_torch as native
    except ImportError:
        return None
    if getattr(native, "built_for", None) != build.built_for():
        return None
    names = []
    for name in ("linear", "linear_input_grad", "linear_weight_grad"):
        names += [name + "_workspace_bytes", name]
    names += ["dropout", "dropout_grad"]
    for name in ("group_norm", "group_norm_grad"):
        names += [name + "_workspace_bytes", name]
    native.use(tuple(C.cast(getattr(L, "qoda_" + n), C.c_void_p).value for n in names))
    return native


def _load():
    global _lib, _native
    if _lib is None:
        L = qoda.load()
        for name in ("linear", "linear_input_grad", "linear_weight_grad", "group_norm", "group_norm_grad"):
            size = getattr(L, f"qoda_{name}_workspace_bytes")
            size.argtypes, size.restype = [C.c_char_p], C.c_int64
            call = getattr(L, f"qoda_{name}")
            call.argtypes, call.restype = [C.c_char_p, C.c_void_p, C.c_size_t, C.c_void_p], C.c_int
        for call in (L.qoda_dropout, L.qoda_dropout_grad):
            call.argtypes, call.restype = [C.c_char_p, C.c_void_p], C.c_int
        L.qoda_operator_error.argtypes, L.qoda_operator_error.restype = [], C.c_char_p
        if _get_device is not None and _get_stream is not None:
            _native = _find_native(L)
        _lib = L
    return _lib


def _is_native() -> bool:
    if _lib is None:
        _load()
    return _native is not None


def _looked_at(call, *args):
    """The native call's outputs; None where its arguments have to be looked at here."""
    global _ready
    if not _ready:
        if not torch.cuda.is_initialized():
            return None
        _ready = True
    device = _get_device()
    out = call(device, _get_stream(device), *args)
    if type(out) is int:
        _raise(out)
    return out


def operator_error() -> str:
    """What the calling thread's last failing operator call found wrong."""
    return _load().qoda_operator_error().decode()


def _raise(code: int):
    raise qoda.QodaError(code, operator_error())


def _run(name: str, args: bytes, device) -> None:
    L = _load()
    need = getattr(L, f"qoda_{name}_workspace_bytes")(args)
    if need < 0:
        _raise(need)
    scratch = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    rc = getattr(L, f"qoda_{name}")(args, scratch.data_ptr() if need else None, need, qoda._stream(None))
    if rc != qoda.OK:
        _raise(rc)


def _on(stream):
    """The stream of a call as a context: allocations and kernels are both on it."""
    return torch.cuda.stream(torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream)


def _activation(name: str) -> int:
    try:
        return ACTIVATIONS[name]
    except (KeyError, TypeError):
        raise ValueError(f"activation {name!r}: one of {', '.join(ACTIVATIONS)}") from None


def _number(activation) -> Optional[int]:
    """For the native look, which takes None for an activation that it does not know."""
    return ACTIVATIONS.get(activation) if isinstance(activation, str) else None


def _first(t: torch.Tensor, name: str) -> int:
    """The type of a call's first tensor."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name}: a CUDA tensor is wanted")
    if t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{name}: the tensor is on device {t.get_device()}, the current device is {torch.cuda.current_device()}")
    dt = DTYPES.get(t.dtype)
    if dt is None:
        raise ValueError(f"{name}: {t.dtype} is neither float32 nor bfloat16")
    if t.dim() == 0:
        raise ValueError(f"{name}: at least one dimension is wanted")
    return dt


def _matrix(t: Optional[torch.Tensor], like: torch.Tensor, name: str, rows: int, cols: int, dtype=None) -> Tuple[int, int]:
    """Address and row stride of a tensor as a matrix of rows x cols, on the device of ``like`` and of its type."""
    if t is None:
        return 0, 0
    if not isinstance(t, torch.Tensor) or t.device != like.device or t.dtype != (dtype or like.dtype):
        raise ValueError(f"{name}: a {dtype or like.dtype} tensor on {like.device} is wanted")
    if t.dim() != 2:
        if t.dim() == 0 or t.shape[-1] != cols:
            raise ValueError(f"{name}: rows of {cols} entries are wanted, the shape is {tuple(t.shape)}")
        try:
            t = t.view(rows, cols)
        except RuntimeError:
            raise ValueError(f"{name}: shape {tuple(t.shape)} with strides {t.stride()} is no matrix of {rows} evenly spaced rows of {cols}") from None
    if t.shape[0] != rows or t.shape[1] != cols:
        raise ValueError(f"{name}: {rows} rows of {cols} entries are wanted, the shape is {tuple(t.shape)}")
    if cols > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: entries of a row have to be adjacent")
    return t.data_ptr(), t.stride(0)


def _vector(t: Optional[torch.Tensor], like: torch.Tensor, name: str, n: int) -> int:
    if t is None:
        return 0
    if not isinstance(t, torch.Tensor) or t.device != like.device or t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name}: {n} contiguous float32 entries on {like.device} are wanted")
    return t.data_ptr()


def _rows(t: torch.Tensor) -> int:
    n = 1
    for s in t.shape[:-1]:
        n *= s
    return n


def _word(v: int, name: str) -> int:
    if not 0 <= v < 1 << 64:
        raise ValueError(f"{name}: {v} is no unsigned 64-bit number")
    return v


class _NotRecorded(torch.autograd.Function):
    """A call's outputs, which raise where torch would differentiate them."""

    @staticmethod
    def forward(ctx, said, call, *inputs):
        ctx.said = said
        return call()

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError(ctx.said)


def _tangents(inputs) -> bool:
    level = torch.autograd.forward_ad
    return level._current_level >= 0 and any(level.unpack_dual(t).tangent is not None for t in inputs)


def _followed(inputs) -> bool:
    """Whether torch is to differentiate by one of a call's inputs."""
    inputs = [t for t in inputs if isinstance(t, torch.Tensor)]
    return _tangents(inputs) or (torch.is_grad_enabled() and any(t.requires_grad for t in inputs))


def _unless_followed(name: str, gradient: str, inputs, call):
    """The outputs of ``call`` if torch is to differentiate by one of its inputs, otherwise None."""
    inputs = [t for t in inputs if isinstance(t, torch.Tensor)]
    said = f"{name} records nothing for torch's differentiation: its gradient is {gradient}"
    if _tangents(inputs):
        raise RuntimeError(said)
    if torch.is_grad_enabled() and any(t.requires_grad for t in inputs):
        return _NotRecorded.apply(said, call, *inputs)
    return None


def linear(x, weight, bias=None, residual=None, *, activation="none", p=0.0, seed=0, offset=0, keep_pre=False, stream=None):
    """residual + drop(act(x weight^T + bias)); with keep_pre also x weight^T + bias, for the gradient of an activation.
    x [..., in], weight [out, in], bias fp32 [out], residual [..., out]."""
    if stream is not None:
        with _on(stream):
            return linear(x, weight, bias, residual, activation=activation, p=p, seed=seed, offset=offset, keep_pre=keep_pre)
    if _is_native():
        out = _looked_at(_native.linear, x, weight, bias, residual, _number(activation), p, seed, offset, keep_pre)
        if out is not None:
            return out
    out = _unless_followed("linear", "linear_input_grad and linear_weight_grad", (x, weight, bias, residual), lambda: linear(
        x, weight, bias, residual, activation=activation, p=p, seed=seed, offset=offset, keep_pre=keep_pre))
    if out is not None:
        return out
    dt, act = _first(x, "linear: x"), _activation(activation)
    if not isinstance(weight, torch.Tensor) or weight.dim() != 2:
        raise ValueError("linear: weight has to be a matrix")
    rows, cin, cout = _rows(x), x.shape[-1], weight.shape[0]
    y = torch.empty(x.shape[:-1] + (cout,), dtype=x.dtype, device=x.device)
    pre = torch.empty_like(y) if keep_pre else None
    _run("linear", _LINEAR.pack(dt, act, rows, cin, cout, *_matrix(x, x, "linear: x", rows, cin), *_matrix(weight, x, "linear: weight", cout, cin),
                                *_matrix(residual, x, "linear: residual", rows, cout), y.data_ptr(), cout, pre.data_ptr() if keep_pre else 0, cout,
                                _vector(bias, x, "linear: bias", cout), p, _word(seed, "seed"), _word(offset, "offset")), x.device)
    return (y, pre) if keep_pre else y


def linear_input_grad(dz, weight, *, pre=None, activation="none", p=0.0, seed=0, offset=0, residual=None, stream=None):
    """residual + drop((dz weight) * act'(pre)): the gradient of linear's x and, with pre, on through the activation and the dropout
    that made x (their pre, p, seed and offset).  dz [..., out], weight [out, in], pre and residual [..., in]."""
    if stream is not None:
        with _on(stream):
            return linear_input_grad(dz, weight, pre=pre, activation=activation, p=p, seed=seed, offset=offset, residual=residual)
    if _is_native():
        out = _looked_at(_native.linear_input_grad, dz, weight, pre, _number(activation), p, seed, offset, residual)
        if out is not None:
            return out
    dt, act = _first(dz, "linear_input_grad: dz"), _activation(activation)
    if not isinstance(weight, torch.Tensor) or weight.dim() != 2:
        raise ValueError("linear_input_grad: weight has to be a matrix")
    rows, cout, cin = _rows(dz), dz.shape[-1], weight.shape[1]
    dx = torch.empty(dz.shape[:-1] + (cin,), dtype=dz.dtype, device=dz.device)
    _run("linear_input_grad", _INPUT_GRAD.pack(
        dt, act, rows, cin, cout, *_matrix(dz, dz, "linear_input_grad: dz", rows, cout), *_matrix(weight, dz, "linear_input_grad: weight", cout, cin),
        *_matrix(pre, dz, "linear_input_grad: pre", rows, cin), *_matrix(residual, dz, "linear_input_grad: residual", rows, cin),
        dx.data_ptr(), cin, p, _word(seed, "seed"), _word(offset, "offset")), dz.device)
    return dx


def linear_weight_grad(dz, x, dweight=None, dbias=None, *, bias=True, accumulate=False, stream=None):
    """(dz^T x, the sum of dz's rows), fp32: written to (or, with accumulate, added to) dweight [out, in] and dbias [out], which are
    made where they are not given.  bias=False: no dbias (None)."""
    if stream is not None:
        with _on(stream):
            return linear_weight_grad(dz, x, dweight, dbias, bias=bias, accumulate=accumulate)
    if _is_native() and isinstance(dz, torch.Tensor) and isinstance(x, torch.Tensor) and dz.is_cuda and dz.dim() > 0 and x.dim() > 0:
        if not accumulate:
            if dweight is None:
                dweight = torch.empty((dz.shape[-1], x.shape[-1]), dtype=torch.float32, device=dz.device)
            if dbias is None and bias:
                dbias = torch.empty(dz.shape[-1], dtype=torch.float32, device=dz.device)
        if (dbias is not None or not bias) and _looked_at(_native.linear_weight_grad, dz, x, dweight, dbias, accumulate) is not None:
            return dweight, dbias
    dt = _first(dz, "linear_weight_grad: dz")
    if not isinstance(x, torch.Tensor) or x.dim() == 0:
        raise ValueError("linear_weight_grad: x has to be a tensor with at least one dimension")
    rows, cout, cin = _rows(dz), dz.shape[-1], x.shape[-1]
    if accumulate and (dweight is None or (bias and dbias is None)):
        raise ValueError("linear_weight_grad: accumulate needs the tensors that are added to")
    if dweight is None:
        dweight = torch.empty((cout, cin), dtype=torch.float32, device=dz.device)
    if dbias is None and bias:
        dbias = torch.empty(cout, dtype=torch.float32, device=dz.device)
    _run("linear_weight_grad", _WEIGHT_GRAD.pack(
        dt, accumulate, rows, cin, cout, *_matrix(dz, dz, "linear_weight_grad: dz", rows, cout), *_matrix(x, dz, "linear_weight_grad: x", rows, cin),
        *_matrix(dweight, dz, "linear_weight_grad: dweight", cout, cin, torch.float32), _vector(dbias, dz, "linear_weight_grad: dbias", cout)), dz.device)
    return dweight, dbias


def _entries(name, call, x, extra, extra_name, activation, p, seed, offset):
    dt, act = _first(x, name), _activation(activation)
    rows, cols = _rows(x), x.shape[-1]
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    rc = call(_DROPOUT.pack(dt, act, rows, cols, *_matrix(x, x, name, rows, cols), *_matrix(extra, x, extra_name, rows, cols), y.data_ptr(), cols,
                            p, _word(seed, "seed"), _word(offset, "offset")), qoda._stream(None))
    if rc != qoda.OK:
        _raise(rc)
    return y


def dropout(x, p, seed, offset, *, activation="none", residual=None, stream=None):
    """residual + drop(act(x))."""
    if stream is not None:
        with _on(stream):
            return dropout(x, p, seed, offset, activation=activation, residual=residual)
    if _is_native():
        out = _looked_at(_native.entries, x, residual, _number(activation), p, seed, offset, False)
        if out is not None:
            return out
    out = _unless_followed("dropout", "dropout_grad", (x, residual), lambda: dropout(x, p, seed, offset, activation=activation, residual=residual))
    if out is not None:
        return out
    return _entries("dropout: x", _load().qoda_dropout, x, residual, "dropout: residual", activation, p, seed, offset)


def dropout_grad(dy, p, seed, offset, *, pre=None, activation="none", stream=None):
    """drop(dy * act'(pre)): the gradient of z in drop(act(z)), pre being z."""
    if stream is not None:
        with _on(stream):
            return dropout_grad(dy, p, seed, offset, pre=pre, activation=activation)
    if _is_native():
        out = _looked_at(_native.entries, dy, pre, _number(activation), p, seed, offset, True)
        if out is not None:
            return out
    return _entries("dropout_grad: dy", _load().qoda_dropout_grad, dy, pre, "dropout_grad: pre", activation, p, seed, offset)


def _values(t: Optional[torch.Tensor], like: torch.Tensor, name: str) -> Tuple[int, int, int]:
    """Address, sample stride and position stride of [samples, ..., channels]."""
    if t is None:
        return 0, 0, 0
    if not isinstance(t, torch.Tensor) or t.device != like.device or t.dtype != like.dtype or t.shape != like.shape:
        raise ValueError(f"{name}: a {like.dtype} tensor of shape {tuple(like.shape)} on {like.device} is wanted")
    n, c = t.shape[0], t.shape[-1]
    if t.dim() != 3:
        positions = 1
        for s in t.shape[1:-1]:
            positions *= s
        try:
            t = t.view(n, positions, c)
        except RuntimeError:
            raise ValueError(f"{name}: the positions of strides {t.stride()} are not evenly spaced") from None
    if c > 1 and t.stride(2) != 1:
        raise ValueError(f"{name}: channels have to be adjacent (channels last)")
    return t.data_ptr(), t.stride(0), t.stride(1)


def _shape(x: torch.Tensor, name: str) -> Tuple[int, int, int]:
    if x.dim() < 2:
        raise ValueError(f"{name}: [samples, ..., channels] is wanted")
    positions = 1
    for s in x.shape[1:-1]:
        positions *= s
    return x.shape[0], positions, x.shape[-1]


def group_norm(x, groups, weight=None, bias=None, *, eps=1e-5, activation="none", stream=None):
    """(act(normalised x * weight + bias), mean, rstd) of x [samples, ..., channels]; mean and rstd [samples, groups], fp32, are what the
    gradient needs (NaN where there is no position or channel).  groups=1 and no position dimensions: the layer normalisation of rows."""
    if stream is not None:
        with _on(stream):
            return group_norm(x, groups, weight, bias, eps=eps, activation=activation)
    if _is_native():
        out = _looked_at(_native.group_norm, x, groups, weight, bias, eps, _number(activation))
        if out is not None:
            return out
    out = _unless_followed("group_norm", "group_norm_grad", (x, weight, bias), lambda: group_norm(x, groups, weight, bias, eps=eps, activation=activation))
    if out is not None:
        return out
    dt, act = _first(x, "group_norm: x"), _activation(activation)
    n, s, c = _shape(x, "group_norm: x")
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    mean = torch.empty((n, max(groups, 0)), dtype=torch.float32, device=x.device)
    rstd = torch.empty_like(mean)
    if s * c == 0:          # the library leaves them alone
        mean.fill_(float("nan"))
        rstd.fill_(float("nan"))
    _run("group_norm", _NORM.pack(dt, act, n, s, c, groups, *_values(x, x, "group_norm: x"), y.data_ptr(), s * c, c,
                                  _vector(weight, x, "group_norm: weight", c), _vector(bias, x, "group_norm: bias", c),
                                  mean.data_ptr(), rstd.data_ptr(), eps), x.device)
    return y, mean, rstd


def group_norm_grad(dy, x, mean, rstd, groups, weight=None, bias=None, *, activation="none", residual=None, dweight=None, dbias=None,
                    accumulate=False, stream=None):
    """(residual + dx, dweight, dbias); dweight and dbias [channels], fp32, are made where they are not given."""
    if stream is not None:
        with _on(stream):
            return group_norm_grad(dy, x, mean, rstd, groups, weight, bias, activation=activation, residual=residual, dweight=dweight, dbias=dbias,
                                   accumulate=accumulate)
    if _is_native() and (not accumulate or (dweight is not None and dbias is not None)):
        out = _looked_at(_native.group_norm_grad, dy, x, mean, rstd, groups, weight, bias, _number(activation), residual, dweight, dbias, accumulate)
        if out is not None:
            return out
    dt, act = _first(x, "group_norm_grad: x"), _activation(activation)
    n, s, c = _shape(x, "group_norm_grad: x")
    if accumulate and (dweight is None or dbias is None):
        raise ValueError("group_norm_grad: accumulate needs the tensors that are added to")
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if dweight is None:
        dweight = torch.empty(c, dtype=torch.float32, device=x.device)
    if dbias is None:
        dbias = torch.empty(c, dtype=torch.float32, device=x.device)
    _run("group_norm_grad", _NORM_GRAD.pack(
        dt, act, n, s, c, groups, *_values(dy, x, "group_norm_grad: dy"), *_values(x, x, "group_norm_grad: x"),
        *_values(residual, x, "group_norm_grad: residual"), dx.data_ptr(), s * c, c,
        _vector(weight, x, "group_norm_grad: weight", c), _vector(bias, x, "group_norm_grad: bias", c),
        _vector(mean, x, "group_norm_grad: mean", n * groups), _vector(rstd, x, "group_norm_grad: rstd", n * groups),
        _vector(dweight, x, "group_norm_grad: dweight", c), _vector(dbias, x, "group_norm_grad: dbias", c), accumulate), x.device)
    return dx, dweight, dbias
