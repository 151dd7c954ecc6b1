"""Thin binding over the operators of include/qoda_matrices.h on torch tensors: matrices in four bits (microscaled: a scale for every 32
entries), products between them and their gradients, and the orthogonalisation of an update by Newton-Schulz products.

Argument marshalling only, as in ``operators``: every operator runs in the library's HIP kernels, and there is no CPU fallback.  Outputs and
scratch memory come from torch's allocator, on the stream that the call runs on (``stream``: a torch stream or a handle; None: the current one).

    wq, wt = microscale(w), microscale(w, transposed=True)                                # once a round
    y, z = mx_linear(x, wq, b, activation="gelu", p=0.1, seed=s, offset=o, keep_pre=True)  # x is rounded in the call
    dz = microscale(dy, rounding="stochastic", seed=s, offset=o)                          # its mean over the draws is dy
    dx = mx_linear_input_grad(dz, wt)
    dzt = microscale(dy, transposed=True, rounding="stochastic", seed=s, offset=o + 1)
    mx_linear_weight_grad(dzt, microscale(x, transposed=True), dweight=g_w, dbias=g_b)    # fp32, into the vector that is quantized
    orthogonalize(g_w, out=g_w)                                                           # ... or its orthogonalised form

An operand of a product has its blocks along what the product sums over, so that a matrix that is summed over both ways is rounded twice.  Plain
rows in a product's first place are rounded to nearest inside the call; up to 16 of them take one launch.  ``activation``, ``p``, ``seed``, ``offset``, ``residual``, biases and
gradients of parameters are as in ``operators``.  Nothing is recorded for torch's differentiation, as there: outputs of ``mx_linear`` on tensors that require a gradient raise where torch asks
for it, and tangents are refused; ``microscale`` and ``orthogonalize``, which have no gradient calls, refuse both at once; what the gradient calls return is plain.
"""
from __future__ import annotations

import ctypes as C
import struct

import torch

from . import operators as ops
from . import qoda

ROUNDINGS = {"nearest": 0, "stochastic": 1}
QUINTIC = (3.4445, -4.7750, 2.0315)       # singular values from 0.002 |g| on come to 0.68 to 1.21 in five steps

# the argument structures of the header, packed as C lays them out
_QUANTIZE = struct.Struct("@3i2q" + "PqPP" + "QQ")
_VALUES = struct.Struct("@i2q" + "PP" + "Pq")
_LINEAR = struct.Struct("@2i3q" + "Pq" + "PP" * 2 + "Pq" * 3 + "PdQQ")
_INPUT_GRAD = struct.Struct("@2i3q" + "Pq" + "PP" * 2 + "Pq" * 3 + "dQQ")
_WEIGHT_GRAD = struct.Struct("@i3q" + "PP" * 2 + "Pq" + "P")
_ORTHOGONALIZE = struct.Struct("@2i3q" + "Pqq" * 2 + "4d")

_lib = None
_native = None          # the native look at the arguments, once the library is loaded


def _load():
    global _lib, _native
    if _lib is None:
        L = ops._load()
        for name in ("mx_linear", "mx_linear_input_grad", "mx_linear_weight_grad", "orthogonalize"):
            size, call = getattr(L, f"qoda_{name}_workspace_bytes"), getattr(L, f"qoda_{name}")
            size.argtypes, size.restype = [C.c_char_p], C.c_int64
            call.argtypes, call.restype = [C.c_char_p, C.c_void_p, C.c_size_t, C.c_void_p], C.c_int
        for call in (L.qoda_mx_quantize, L.qoda_mx_values):
            call.argtypes, call.restype = [C.c_char_p, C.c_void_p], C.c_int
        for size in (L.qoda_mx_code_bytes, L.qoda_mx_scale_bytes):
            size.argtypes, size.restype = [C.c_int64, C.c_int64], C.c_int64
        if ops._native is not None:
            names = ["mx_quantize", "mx_values"]
            for name in ("mx_linear", "mx_linear_input_grad", "mx_linear_weight_grad", "orthogonalize"):
                names += [name + "_workspace_bytes", name]
            ops._native.use_matrices(tuple(C.cast(getattr(L, "qoda_" + n), C.c_void_p).value for n in names))
            _native = ops._native
        _lib = L
    return _lib


def _is_native() -> bool:
    if _lib is None:
        _load()
    return _native is not None


def _on(stream):
    return ops._on(stream)


def _shapes(rows: int, cols: int):
    """Of the codes and of the scales of a microscaled matrix."""
    steps = -(-cols // 256)
    return (rows, 128 * steps), (2 * steps, -(-rows // 64), 256)


def _bytes(t, shape, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.uint8 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"Microscaled: {name} are a contiguous uint8 tensor of shape {shape}")
    return t


class Microscaled:
    """A matrix of rows x cols in four bits, rounded by ``microscale`` or laid out by the caller as include/qoda_matrices.h says: ``codes`` and ``scales``
    are contiguous uint8 tensors on one device, [rows, 128 s] and [2 s, rows / 64 rounded up, 256], s = cols / 256 rounded up."""

    __slots__ = ("_parts",)

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, rows: int, cols: int):
        self._parts = (_bytes(codes, (rows, (cols + 255) // 256 * 128), "codes"), _bytes(scales, ((cols + 255) // 256 * 2, (rows + 63) // 64, 256), "scales"), rows, cols)
        if codes.device != scales.device:
            raise ValueError("Microscaled: codes and scales are on different devices")

    @property
    def codes(self) -> torch.Tensor:
        return self._apart()[0]

    @property
    def scales(self) -> torch.Tensor:
        return self._apart()[1]

    def _apart(self):
        """(codes, scales, rows, columns), where one tensor holds both so far."""
        both, scales, rows, cols = self._parts
        if scales is None:
            of_codes, of_scales = _shapes(rows, cols)
            n = of_codes[0] * of_codes[1]
            self._parts = (both[:n].view(of_codes), both[n:].view(of_scales), rows, cols)
        return self._parts

    rows = property(lambda self: self._parts[2])
    cols = property(lambda self: self._parts[3])
    shape = property(lambda self: torch.Size(self._parts[2:]))
    device = property(lambda self: self._parts[0].device)

    def values(self, dtype=torch.float32, *, stream=None) -> torch.Tensor:
        """What the codes stand for, a matrix of float32 or bfloat16."""
        if stream is not None:
            with _on(stream):
                return self.values(dtype)
        if _native is not None or _is_native():
            out = ops._looked_at(_native.mx_values, self._parts, _bf16(dtype))
            if out is not None:
                return out
        dt = _type(dtype, "values")
        _current(self, "values")
        y = torch.empty((self.rows, self.cols), dtype=dtype, device=self.device)
        _call("mx_values", _VALUES.pack(dt, self.rows, self.cols, *_mx(self), y.data_ptr(), self.cols))
        return y

    def __repr__(self) -> str:
        return f"Microscaled({self.rows} x {self.cols}, {self.device})"


_new = object.__new__


def _bf16(dtype):
    """For the native look, which takes None for a type that it does not know."""
    return True if dtype is torch.bfloat16 else False if dtype is torch.float32 else None


def _plain_or_parts(x, dtype):
    """A product's first operand and its type, for the native look."""
    if type(x) is Microscaled:
        return x._parts, True if dtype is None else _bf16(dtype)
    return x, None if dtype is None or (isinstance(x, torch.Tensor) and dtype is x.dtype) else False


def _parts(q):
    return q._parts if type(q) is Microscaled else None


def _mx(q):
    return q.codes.data_ptr(), q.scales.data_ptr()


def _type(dtype, name: str) -> int:
    dt = ops.DTYPES.get(dtype)
    if dt is None:
        raise ValueError(f"{name}: {dtype} is neither float32 nor bfloat16")
    return dt


def _current(q: Microscaled, name: str) -> None:
    if q.device.type != "cuda":
        raise ValueError(f"{name}: a CUDA tensor is wanted")
    if q.device.index != torch.cuda.current_device():
        raise ValueError(f"{name}: the matrix is on {q.device}, the current device is {torch.cuda.current_device()}")


def _microscaled(q, name: str, rows: int, cols: int, device) -> Microscaled:
    if not isinstance(q, Microscaled):
        raise ValueError(f"{name}: a Microscaled matrix is wanted")
    if q.rows != rows or q.cols != cols:
        raise ValueError(f"{name}: {rows} rows of {cols} entries are wanted, the matrix has {q.rows} of {q.cols}")
    if q.device != device:
        raise ValueError(f"{name}: the matrix is on {q.device}, the others on {device}")
    return q


def _call(name: str, args: bytes) -> None:
    rc = getattr(_load(), f"qoda_{name}")(args, qoda._stream(None))
    if rc != qoda.OK:
        ops._raise(rc)


def _run(name: str, args: bytes, device) -> None:
    _load()
    ops._run(name, args, device)


def microscale(x, *, transposed=False, rounding="nearest", seed=0, offset=0, stream=None) -> Microscaled:
    """The matrix x [..., columns] (the dimensions before the last are rows) in four bits or, with transposed, its transpose.  rounding: "nearest", or
    "stochastic": an entry goes to the neighbour above or below by a draw that (seed, offset, its place in the result) fixes, and in the mean stays
    what it is."""
    if stream is not None:
        with _on(stream):
            return microscale(x, transposed=transposed, rounding=rounding, seed=seed, offset=offset)
    if rounding.__class__ is not str or rounding not in ROUNDINGS:
        raise ValueError(f"rounding {rounding!r}: one of {', '.join(ROUNDINGS)}")
    if _native is not None or _is_native():
        out = ops._looked_at(_native.microscale, x, transposed, rounding == "stochastic", seed, offset)
        if out is not None:
            q = _new(Microscaled)
            q._parts = out
            return q
    if ops._followed((x,)):
        raise RuntimeError("microscale: rounding has no derivative, and nothing is recorded for torch's differentiation; x.detach() is rounded")
    dt = ops._first(x, "microscale: x")
    rows, cols = ops._rows(x), x.shape[-1]
    at, stride = ops._matrix(x, x, "microscale: x", rows, cols)
    codes, scales = _shapes(cols, rows) if transposed else _shapes(rows, cols)
    q = Microscaled(torch.empty(codes, dtype=torch.uint8, device=x.device), torch.empty(scales, dtype=torch.uint8, device=x.device),
                    *((cols, rows) if transposed else (rows, cols)))
    _call("mx_quantize", _QUANTIZE.pack(dt, bool(transposed), ROUNDINGS[rounding], rows, cols, at, stride, *_mx(q), ops._word(seed, "seed"),
                                        ops._word(offset, "offset")))
    return q


def _first(x, name: str, dtype):
    """(the type of the call, the type of its entries, rows, columns, shape before the columns, its place as plain rows, and as a microscaled matrix)"""
    if isinstance(x, Microscaled):
        dtype = torch.bfloat16 if dtype is None else dtype
        dt = _type(dtype, name)
        _current(x, name)
        return dt, dtype, x.rows, x.cols, (x.rows,), (0, 0), _mx(x)
    dt = ops._first(x, name)
    if dtype is not None and dtype != x.dtype:
        raise ValueError(f"{name}: dtype is that of the rows, {x.dtype}")
    rows, cols = ops._rows(x), x.shape[-1]
    return dt, x.dtype, rows, cols, tuple(x.shape[:-1]), ops._matrix(x, x, name, rows, cols), (0, 0)


def mx_linear(x, weight, bias=None, residual=None, *, activation="none", p=0.0, seed=0, offset=0, keep_pre=False, dtype=None, stream=None):
    """residual + drop(act(x weight^T + bias)); with keep_pre also x weight^T + bias, for the gradient of an activation.
    x [..., in], plain or Microscaled, weight Microscaled [out, in], bias fp32 [out], residual [..., out].  dtype: of the outputs where x is
    Microscaled (bfloat16 if it is not given); otherwise they have x's."""
    if stream is not None:
        with _on(stream):
            return mx_linear(x, weight, bias, residual, activation=activation, p=p, seed=seed, offset=offset, keep_pre=keep_pre, dtype=dtype)
    if _native is not None or _is_native():
        first, bf16 = _plain_or_parts(x, dtype)
        out = ops._looked_at(_native.mx_linear, first, _parts(weight), bias, residual, ops._number(activation), p, seed, offset, keep_pre, bf16)
        if out is not None:
            return out
    out = ops._unless_followed("mx_linear", "mx_linear_input_grad and mx_linear_weight_grad", (x, bias, residual), lambda: mx_linear(
        x, weight, bias, residual, activation=activation, p=p, seed=seed, offset=offset, keep_pre=keep_pre, dtype=dtype))
    if out is not None:
        return out
    dt, dtype, rows, cin, front, plain, xq = _first(x, "mx_linear: x", dtype)
    act = ops._activation(activation)
    if not isinstance(weight, Microscaled):
        raise ValueError("mx_linear: weight: a Microscaled matrix is wanted")
    cout = weight.rows
    _microscaled(weight, "mx_linear: weight", cout, cin, x.device)
    y = torch.empty(front + (cout,), dtype=dtype, device=x.device)
    pre = torch.empty_like(y) if keep_pre else None
    _run("mx_linear", _LINEAR.pack(dt, act, rows, cin, cout, *plain, *xq, *_mx(weight), *ops._matrix(residual, y, "mx_linear: residual", rows, cout),
                                   y.data_ptr(), cout, pre.data_ptr() if keep_pre else 0, cout, ops._vector(bias, y, "mx_linear: bias", cout), p,
                                   ops._word(seed, "seed"), ops._word(offset, "offset")), x.device)
    return (y, pre) if keep_pre else y


def mx_linear_input_grad(dz, weight_t, *, pre=None, activation="none", p=0.0, seed=0, offset=0, residual=None, dtype=None, stream=None):
    """residual + drop((dz weight) * act'(pre)), as operators.linear_input_grad.  dz [..., out], plain or Microscaled; weight_t: the weight's transpose,
    Microscaled [in, out]; pre and residual [..., in]; dtype as in mx_linear."""
    if stream is not None:
        with _on(stream):
            return mx_linear_input_grad(dz, weight_t, pre=pre, activation=activation, p=p, seed=seed, offset=offset, residual=residual, dtype=dtype)
    if _native is not None or _is_native():
        first, bf16 = _plain_or_parts(dz, dtype)
        out = ops._looked_at(_native.mx_linear_input_grad, first, _parts(weight_t), pre, ops._number(activation), p, seed, offset, residual, bf16)
        if out is not None:
            return out
    dt, dtype, rows, cout, front, plain, dzq = _first(dz, "mx_linear_input_grad: dz", dtype)
    act = ops._activation(activation)
    if not isinstance(weight_t, Microscaled):
        raise ValueError("mx_linear_input_grad: weight_t: a Microscaled matrix is wanted")
    cin = weight_t.rows
    _microscaled(weight_t, "mx_linear_input_grad: weight_t", cin, cout, dz.device)
    dx = torch.empty(front + (cin,), dtype=dtype, device=dz.device)
    _run("mx_linear_input_grad", _INPUT_GRAD.pack(
        dt, act, rows, cin, cout, *plain, *dzq, *_mx(weight_t), *ops._matrix(pre, dx, "mx_linear_input_grad: pre", rows, cin),
        *ops._matrix(residual, dx, "mx_linear_input_grad: residual", rows, cin), dx.data_ptr(), cin, p, ops._word(seed, "seed"), ops._word(offset, "offset")),
        dz.device)
    return dx


def mx_linear_weight_grad(dz_t, x_t, dweight=None, dbias=None, *, bias=True, accumulate=False, stream=None):
    """(dz_t x_t^T, the sums of dz_t's rows), fp32: written to (or, with accumulate, added to) dweight [out, in] and dbias [out], which are
    made where they are not given.  dz_t [out, rows] and x_t [in, rows] are Microscaled: the transposes of dz and x.  bias=False: no dbias (None)."""
    if stream is not None:
        with _on(stream):
            return mx_linear_weight_grad(dz_t, x_t, dweight, dbias, bias=bias, accumulate=accumulate)
    if _is_native() and type(dz_t) is Microscaled and type(x_t) is Microscaled and dz_t._parts[0].is_cuda and not (accumulate and (dweight is None or (bias and dbias is None))):
        if dweight is None:
            dweight = torch.empty((dz_t.rows, x_t.rows), dtype=torch.float32, device=dz_t.device)
        if dbias is None and bias:
            dbias = torch.empty(dz_t.rows, dtype=torch.float32, device=dz_t.device)
        if ops._looked_at(_native.mx_linear_weight_grad, dz_t._parts, x_t._parts, dweight, dbias, accumulate) is not None:
            return dweight, dbias
    for q, name in ((dz_t, "dz_t"), (x_t, "x_t")):
        if not isinstance(q, Microscaled):
            raise ValueError(f"mx_linear_weight_grad: {name}: a Microscaled matrix is wanted")
    _current(dz_t, "mx_linear_weight_grad: dz_t")
    cout, cin, rows = dz_t.rows, x_t.rows, dz_t.cols
    _microscaled(x_t, "mx_linear_weight_grad: x_t", cin, rows, dz_t.device)
    if accumulate and (dweight is None or (bias and dbias is None)):
        raise ValueError("mx_linear_weight_grad: accumulate needs the tensors that are added to")
    if dweight is None:
        dweight = torch.empty((cout, cin), dtype=torch.float32, device=dz_t.device)
    if dbias is None and bias:
        dbias = torch.empty(cout, dtype=torch.float32, device=dz_t.device)
    _run("mx_linear_weight_grad", _WEIGHT_GRAD.pack(
        bool(accumulate), rows, cin, cout, *_mx(dz_t), *_mx(x_t), *ops._matrix(dweight, dz_t.codes, "mx_linear_weight_grad: dweight", cout, cin, torch.float32),
        ops._vector(dbias, dz_t.codes, "mx_linear_weight_grad: dbias", cout)), dz_t.device)
    return dweight, dbias

def _matrices(t: torch.Tensor, like: torch.Tensor, name: str):
    """Address, strides of matrices and rows, of [..., rows, columns]."""
    if not isinstance(t, torch.Tensor) or t.device != like.device or t.dtype != like.dtype or t.shape != like.shape:
        raise ValueError(f"{name}: a {like.dtype} tensor of shape {tuple(like.shape)} on {like.device} is wanted")
    n = 1
    for d in t.shape[:-2]:
        n *= d
    try:
        t = t.view(n, *t.shape[-2:])
    except RuntimeError:
        raise ValueError(f"{name}: the matrices of strides {t.stride()} are not evenly spaced") from None
    if t.shape[2] > 1 and t.stride(2) != 1:
        raise ValueError(f"{name}: entries of a row have to be adjacent")
    return t.data_ptr(), t.stride(0), t.stride(1)


def orthogonalize(g, *, steps=5, coefficients=QUINTIC, eps=1e-7, out=None, stream=None):
    """The matrices g [..., rows, columns] with their singular values brought towards 1: X = g / (|g| + eps), then ``steps`` times (1000 at most)
    X <- a X + (b A + c A A) X with A = X X^T and (a, b, c) = coefficients.  Written to out, if given, which may be g (or apart from it); of g's type."""
    if stream is not None:
        with _on(stream):
            return orthogonalize(g, steps=steps, coefficients=coefficients, eps=eps, out=out)
    a, b, c = coefficients
    if _native is not None or _is_native():
        x = ops._looked_at(_native.orthogonalize, g, steps, a, b, c, eps, out)
        if x is not None:
            return x
    if ops._followed((g, out)):
        raise RuntimeError("orthogonalize records nothing for torch's differentiation; g.detach() is orthogonalised")
    dt = ops._first(g, "orthogonalize: g")
    if g.dim() < 2:
        raise ValueError("orthogonalize: g: [..., rows, columns] is wanted")
    n, (rows, cols) = 1, g.shape[-2:]
    for d in g.shape[:-2]:
        n *= d
    x = torch.empty(g.shape, dtype=g.dtype, device=g.device) if out is None else out
    _run("orthogonalize", _ORTHOGONALIZE.pack(dt, steps, n, rows, cols, *_matrices(g, g, "orthogonalize: g"), *_matrices(x, g, "orthogonalize: out"),
                                              a, b, c, eps), g.device)
    return x
