"""include/qoda_matrices.h without a GPU: exported names, the packed argument structures, sizes and refusals."""
import os
import re
import shutil
import struct
import subprocess

import pytest

from paper_2505_14371_amd import matrices as mats
from paper_2505_14371_amd import qoda

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "qoda_matrices.h")
STRUCTS = {"qoda_mx_quantize_args": ("_QUANTIZE", "offset"), "qoda_mx_values_args": ("_VALUES", "y"), "qoda_mx_linear_args": ("_LINEAR", "offset"),
           "qoda_mx_linear_input_grad_args": ("_INPUT_GRAD", "offset"), "qoda_mx_linear_weight_grad_args": ("_WEIGHT_GRAD", "dbias"),
           "qoda_orthogonalize_args": ("_ORTHOGONALIZE", "eps")}


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(qoda.LIB_PATH):
        from paper_2505_14371_amd import build

        build.build()
    return mats._load()


def test_library_exports_every_declared_call(lib):
    names = set(re.findall(r"\b(qoda_[a-z_]+)\s*\(", re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)))
    assert len(names) >= 10
    for name in names:
        assert hasattr(lib, name), name


def test_packed_arguments_have_the_structures_layout(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "layout.c"
    src.write_text('#include "qoda_matrices.h"\n#include <stdio.h>\nint main(void) {\n' + "".join(
        f'printf("%zu %zu\\n", sizeof({n}), offsetof({n}, {last}));\n' for n, (_, last) in STRUCTS.items()) + "return 0; }\n")
    subprocess.check_call([gcc, "-I" + os.path.dirname(HEADER), str(src), "-o", str(tmp_path / "layout")])
    lines = subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.split("\n")
    for (name, (packed, last)), line in zip(STRUCTS.items(), lines):
        s = getattr(mats, packed)
        size, at = (int(v) for v in line.split())
        assert s.size == size, name
        fields = re.sub(r"(\d+)([a-zA-Z])", lambda m: m.group(2) * int(m.group(1)), s.format[1:])
        tail = 2 if last == "y" else 1          # a matrix: address and stride
        assert struct.calcsize("@" + fields[:-tail] + "0" + fields[-tail]) == at, name


def test_sizes_of_microscaled_matrices(lib):
    for rows, cols, codes, scales in ((0, 0, 0, 0), (1, 1, 128, 512), (64, 256, 64 * 128, 512), (65, 257, 65 * 256, 2048), (0x7FFF0000, 8192, 0x7FFF0000 * 4096, 0x7FFF0000 * 256)):
        assert lib.qoda_mx_code_bytes(rows, cols) == codes and lib.qoda_mx_scale_bytes(rows, cols) == scales
        c, s = mats._shapes(rows, cols)
        assert c[0] * c[1] == codes and s[0] * s[1] * s[2] == scales
    for rows, cols in ((-1, 4), (4, -1), (0x7FFF0001, 1), (1, 1 << 40)):
        assert lib.qoda_mx_code_bytes(rows, cols) == qoda.EINVAL and lib.qoda_mx_scale_bytes(rows, cols) == qoda.EINVAL


A = 4096            # an address that is never followed: every call below is refused, or has nothing to do


def quantize(dtype=0, transposed=0, stochastic=0, rows=4, cols=8, x=A, xs=8, codes=A, scales=A):
    return "mx_quantize", mats._QUANTIZE.pack(dtype, transposed, stochastic, rows, cols, x, xs, codes, scales, 0, 0)


def values(dtype=0, rows=4, cols=8, codes=A, scales=A, y=A, ys=8):
    return "mx_values", mats._VALUES.pack(dtype, rows, cols, codes, scales, y, ys)


def linear(dtype=0, act=0, rows=4, cin=8, cout=6, x=A, xs=8, xc=0, xsc=0, wc=A, wsc=A, r=0, rs=6, y=A, ys=6, z=0, zs=6, bias=0, p=0.0):
    return "mx_linear", mats._LINEAR.pack(dtype, act, rows, cin, cout, x, xs, xc, xsc, wc, wsc, r, rs, y, ys, z, zs, bias, p, 0, 0)


def input_grad(dtype=0, act=0, rows=4, cin=8, cout=6, dz=A, dzs=6, dc=0, dsc=0, wc=A, wsc=A, z=0, zs=8, r=0, rs=8, dx=A, dxs=8, p=0.0):
    return "mx_linear_input_grad", mats._INPUT_GRAD.pack(dtype, act, rows, cin, cout, dz, dzs, dc, dsc, wc, wsc, z, zs, r, rs, dx, dxs, p, 0, 0)


def weight_grad(rows=4, cin=8, cout=6, dc=A, dsc=A, xc=A, xsc=A, dw=A, dws=8, db=0):
    return "mx_linear_weight_grad", mats._WEIGHT_GRAD.pack(0, rows, cin, cout, dc, dsc, xc, xsc, dw, dws, db)


def orthogonalize(dtype=0, steps=5, n=2, rows=4, cols=6, g=A, gm=24, gr=6, x=A, xm=24, xr=6, a=3.4445, b=-4.7750, c=2.0315, eps=1e-7):
    return "orthogonalize", mats._ORTHOGONALIZE.pack(dtype, steps, n, rows, cols, g, gm, gr, x, xm, xr, a, b, c, eps)


BIG, INF, NAN = (1 << 24) + 1, float("inf"), float("nan")
REFUSED = [
    (quantize(dtype=2), "dtype 2"), (quantize(rows=-1), "size of -1"), (quantize(cols=1 << 31), "size of"), (quantize(x=0), "x is null"), (quantize(x=A + 2), "x is not aligned"),
    (quantize(xs=7), "stride of 7"), (quantize(codes=0), "q is null"), (quantize(scales=0), "q is null"), (quantize(codes=A + 8), "16 bytes"), (quantize(scales=A + 4), "16 bytes"),
    (values(dtype=-1), "dtype -1"), (values(rows=-5), "size"), (values(codes=0), "q is null"), (values(scales=A + 1), "16 bytes"), (values(y=0), "y is null"), (values(ys=3), "stride"),
    (linear(dtype=3), "dtype"), (linear(act=5), "activation 5"), (linear(act=-1), "activation"), (linear(rows=-1), "size"), (linear(cin=BIG, xs=BIG), "sums over"), (linear(p=1.5), "p = 1.5"),
    (linear(p=float("nan")), "p = "), (linear(x=0), "x is null"), (linear(x=0, xc=A), "x is null"), (linear(x=0, xc=A + 1, xsc=A), "16 bytes"), (linear(xs=2), "stride of 2"),
    (linear(wc=0), "w is null"), (linear(wsc=A + 3), "16 bytes"), (linear(r=A + 1), "residual is not aligned"), (linear(r=A, rs=1), "residual has a stride"), (linear(y=0), "y is null"),
    (linear(z=A, zs=5), "pre has a stride"), (linear(bias=A + 2), "bias is not aligned"),
    (input_grad(dtype=9), "dtype"), (input_grad(act=1), "pre is null"), (input_grad(cout=BIG, dzs=BIG), "sums over"), (input_grad(dz=0), "dz is null"), (input_grad(dz=A + 1), "dz is not aligned"),
    (input_grad(wc=0), "wt is null"), (input_grad(dx=0), "dx is null"), (input_grad(dxs=1), "dx has a stride"), (input_grad(r=A, rs=2), "residual has a stride"), (input_grad(p=-0.1), "p = "),
    (weight_grad(rows=BIG), "sums over"), (weight_grad(rows=-1), "size"), (weight_grad(dc=0), "dzt is null"), (weight_grad(xsc=0), "xt is null"), (weight_grad(xc=A + 8), "16 bytes"),
    (weight_grad(dw=0), "dw is null"), (weight_grad(dw=A + 2), "dw is not aligned"), (weight_grad(dws=7), "stride of 7"), (weight_grad(db=A + 1), "dbias is not aligned"),
    (orthogonalize(dtype=7), "dtype 7"), (orthogonalize(steps=-1), "-1 steps"), (orthogonalize(steps=1001), "1001 steps"), (orthogonalize(steps=1000, a=1.03, b=0.0, c=0.0), "2^40"), (orthogonalize(n=-1), "size"), (orthogonalize(eps=-1e-9), "eps"), (orthogonalize(eps=NAN), "eps"), (orthogonalize(eps=INF), "eps"),
    (orthogonalize(a=NAN), "coefficients"), (orthogonalize(b=INF), "coefficients"), (orthogonalize(a=1e13), "2^40"), (orthogonalize(a=10.0, b=0.0, c=0.0, steps=13), "2^40"),
    (orthogonalize(b=1e30, c=-1e30), "2^40"), (orthogonalize(g=0), "g is null"), (orthogonalize(x=0), "x is null"), (orthogonalize(g=A + 2), "g is not aligned"), (orthogonalize(xr=5), "strides of x"),
    (orthogonalize(gm=23), "strides of g"), (orthogonalize(gm=-24), "strides of g"), (orthogonalize(rows=(1 << 17) + 1, cols=(1 << 17) + 1, gr=1 << 18, gm=1 << 36, xr=1 << 18, xm=1 << 36), "sides"),
    (orthogonalize(rows=1, cols=(1 << 22) + 1), "sides"),
]


def call(lib, name, args, workspace=None, have=0):
    if name in ("mx_quantize", "mx_values"):
        return getattr(lib, "qoda_" + name)(args, None)
    return getattr(lib, "qoda_" + name)(args, workspace, have, None)


@pytest.mark.parametrize("at", range(len(REFUSED)))
def test_refusals(lib, at):
    (name, args), said = REFUSED[at]
    assert call(lib, name, args) == qoda.EINVAL
    text = lib.qoda_operator_error().decode()
    assert said in text and text.startswith("qoda_" + name), text
    if name not in ("mx_quantize", "mx_values"):
        assert getattr(lib, f"qoda_{name}_workspace_bytes")(args) == qoda.EINVAL


def test_null_arguments(lib):
    for name in ("mx_quantize", "mx_values", "mx_linear", "mx_linear_input_grad", "mx_linear_weight_grad", "orthogonalize"):
        assert call(lib, name, None) == qoda.EINVAL and "null" in lib.qoda_operator_error().decode()


@pytest.mark.parametrize("args", [quantize(rows=0, x=0, codes=0), quantize(cols=0, x=0, scales=0), values(rows=0, codes=0, y=0), linear(rows=0, x=0, y=0, wc=0), linear(cout=0, y=0, wc=0),
                                  input_grad(rows=0, dz=0, dx=0), input_grad(cin=0, dx=0), weight_grad(cout=0, dw=0, dc=0), weight_grad(cin=0, xc=0, dw=0),
                                  orthogonalize(n=0, g=0), orthogonalize(rows=0, x=0), orthogonalize(cols=0, g=0, x=0)])
def test_empty_outputs_need_nothing(lib, args):
    assert call(lib, *args) == qoda.OK, lib.qoda_operator_error()


def test_too_small_a_workspace_is_refused(lib):
    name, args = linear(rows=100, cin=600, cout=6, xs=600)
    need = lib.qoda_mx_linear_workspace_bytes(args)
    assert need >= lib.qoda_mx_code_bytes(100, 600) + lib.qoda_mx_scale_bytes(100, 600)
    for workspace, have in ((None, need), (A, need - 1), (A + 8, need)):
        assert call(lib, name, args, workspace, have) == qoda.EINVAL and "workspace" in lib.qoda_operator_error().decode()
    name, args = weight_grad(rows=100000, cin=64, cout=64, dws=64)
    need = lib.qoda_mx_linear_weight_grad_workspace_bytes(args)
    assert need > 0 and need % (64 * 64 * 4) == 0 and call(lib, name, args, A, need - 4) == qoda.EINVAL


def test_arguments_that_python_refuses(lib):
    u8 = lambda *shape: torch.zeros(shape, dtype=torch.uint8)  # noqa: E731
    q = mats.Microscaled(u8(5, 256), u8(4, 1, 256), 5, 300)
    assert q.shape == (5, 300) and "5 x 300" in repr(q)
    for codes, scales in ((u8(5, 128), u8(4, 1, 256)), (u8(5, 256), u8(2, 1, 256)), (u8(5, 256).int(), u8(4, 1, 256)), (u8(256, 5).t(), u8(4, 1, 256)), (None, u8(4, 1, 256))):
        with pytest.raises(ValueError):
            mats.Microscaled(codes, scales, 5, 300)
    for bad in (lambda: q.values(), lambda: mats.mx_linear(q, q), lambda: mats.microscale(torch.zeros(3, 4)), lambda: mats.mx_linear_weight_grad(q, q), lambda: mats.mx_linear_weight_grad(1, q),
                lambda: mats.mx_linear_input_grad(torch.zeros(3, 4), q), lambda: q.values(torch.float16), lambda: mats.microscale(torch.zeros(3, 4), rounding="up"),
                lambda: mats.microscale(torch.zeros(3, 4), rounding=[])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(RuntimeError, match="no derivative"):
        mats.microscale(torch.zeros(3, 4, requires_grad=True))


def test_bounded_polynomials_are_taken(lib):
    wide = dict(rows=300, cols=400, gr=400, gm=120000, xr=400, xm=120000)
    for steps in (0, 1, 1000):
        assert lib.qoda_orthogonalize_workspace_bytes(orthogonalize(steps=steps, **wide)[1]) > 0
    assert lib.qoda_orthogonalize_workspace_bytes(orthogonalize(a=10.0, b=0.0, c=0.0, steps=12, **wide)[1]) > 0
    assert lib.qoda_orthogonalize_workspace_bytes(orthogonalize()[1]) == 0          # small ones stay in shared memory
    name, args = orthogonalize(**wide)
    need = lib.qoda_orthogonalize_workspace_bytes(args)
    assert call(lib, name, args, A, need - 1) == qoda.EINVAL and "workspace" in lib.qoda_operator_error().decode()
