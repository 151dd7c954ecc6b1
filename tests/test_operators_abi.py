"""include/qoda_operators.h without a GPU: exported names, the packed argument structures, refusals, the generator's words."""
import ctypes
import os
import re
import shutil
import struct
import subprocess

import numpy as np
import pytest

import operator_definitions as D
from paper_2505_14371_amd import operators as ops
from paper_2505_14371_amd import qoda

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "qoda_operators.h")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(qoda.LIB_PATH):
        from paper_2505_14371_amd import build

        build.build()
    return ops._load()


def test_library_exports_every_declared_call(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(qoda_[a-z_]+)\s*\(", text))
    assert len(names) == 13
    for name in names:
        assert hasattr(lib, name), name
    for name in ("linear", "linear_input_grad", "linear_weight_grad", "dropout", "dropout_grad", "group_norm", "group_norm_grad", "operator_error"):
        assert callable(getattr(ops, name)) and f"qoda_{name}" in names


def test_packed_arguments_have_the_structures_layout(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    packed = {"qoda_linear_args": ops._LINEAR, "qoda_linear_input_grad_args": ops._INPUT_GRAD, "qoda_linear_weight_grad_args": ops._WEIGHT_GRAD,
              "qoda_dropout_args": ops._DROPOUT, "qoda_group_norm_args": ops._NORM, "qoda_group_norm_grad_args": ops._NORM_GRAD}
    last = {"qoda_linear_args": "offset", "qoda_linear_input_grad_args": "offset", "qoda_linear_weight_grad_args": "dbias", "qoda_dropout_args": "offset",
            "qoda_group_norm_args": "eps", "qoda_group_norm_grad_args": "accumulate"}
    src = tmp_path / "layout.c"
    src.write_text('#include "qoda_operators.h"\n#include <stdio.h>\nint main(void) {\n' + "".join(
        f'printf("%zu %zu\\n", sizeof({n}), offsetof({n}, {last[n]}));\n' for n in packed) + "return 0; }\n")
    subprocess.check_call([gcc, "-I" + os.path.dirname(HEADER), str(src), "-o", str(tmp_path / "layout")])
    lines = subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.split("\n")
    for (name, s), line in zip(packed.items(), lines):
        size, at = (int(v) for v in line.split())
        assert s.size == size, name
        fields = re.sub(r"(\d+)([a-zA-Z])", lambda m: m.group(2) * int(m.group(1)), s.format[1:])
        assert struct.calcsize("@" + fields[:-1] + "0" + fields[-1]) == at, name


def linear(dtype=0, act=0, rows=4, cin=8, cout=6, x=4096, xs=8, w=4096, ws=8, r=0, rs=6, y=8192, ys=6, z=0, zs=6, bias=0, p=0.0):
    return ops._LINEAR.pack(dtype, act, rows, cin, cout, x, xs, w, ws, r, rs, y, ys, z, zs, bias, p, 0, 0)


def test_refusals_launch_nothing(lib):
    """Each is refused before the device is touched: the addresses are none."""
    bad = [(dict(dtype=2), b"dtype"), (dict(dtype=-1), b"dtype"), (dict(act=5), b"activation"), (dict(rows=-1), b"size"), (dict(cin=1 << 31), b"size"),
           (dict(x=0), b"x is null"), (dict(w=0), b"w is null"), (dict(y=0), b"y is null"), (dict(x=4097), b"x is not aligned"), (dict(dtype=1, w=4097), b"w is not aligned"),
           (dict(xs=7), b"x has a stride"), (dict(ws=-8), b"w has a stride"), (dict(ys=5), b"y has a stride"), (dict(z=4096, zs=5), b"pre has a stride"),
           (dict(r=4096, rs=0), b"residual has a stride"), (dict(bias=4098), b"bias"), (dict(p=-0.1), b"p ="), (dict(p=1.01), b"p ="), (dict(p=float("nan")), b"p =")]
    for kw, said in bad:
        a = linear(**kw)
        assert lib.qoda_linear(a, None, 0, None) == qoda.EINVAL, kw
        assert said in lib.qoda_operator_error(), (kw, lib.qoda_operator_error())
        assert lib.qoda_linear_workspace_bytes(a) == qoda.EINVAL
    for call in (lib.qoda_linear, lib.qoda_linear_input_grad, lib.qoda_linear_weight_grad, lib.qoda_group_norm, lib.qoda_group_norm_grad):
        assert call(None, None, 0, None) == qoda.EINVAL and b"null" in lib.qoda_operator_error()
    assert lib.qoda_dropout(None, None) == lib.qoda_dropout_grad(None, None) == qoda.EINVAL
    grad = lambda act, z: ops._INPUT_GRAD.pack(0, act, 4, 8, 6, 4096, 6, 4096, 8, z, 8, 0, 8, 8192, 8, 0.0, 0, 0)  # noqa: E731
    assert lib.qoda_linear_input_grad(grad(3, 0), None, 0, None) == qoda.EINVAL and b"pre is null" in lib.qoda_operator_error()
    norm = lambda n=2, s=3, c=8, g=2, x=4096, xn=24, xp=8, eps=1e-5, mean=4096: ops._NORM.pack(0, 0, n, s, c, g, x, xn, xp, 8192, 24, 8, 0, 0, mean, 4096, eps)  # noqa: E731
    for kw, said in ((dict(g=3), b"divide"), (dict(g=0), b"divide"), (dict(xp=7), b"strides of x"), (dict(xn=23), b"strides of x"), (dict(x=0), b"x is null"),
                     (dict(eps=-1.0), b"eps"), (dict(eps=float("inf")), b"eps"), (dict(mean=0), b"mean"), (dict(n=1 << 30, xn=24), b"2^31")):
        assert lib.qoda_group_norm(norm(**kw), None, 0, None) == qoda.EINVAL, kw
        assert said in lib.qoda_operator_error(), (kw, lib.qoda_operator_error())


def test_empty_outputs_are_no_error(lib):
    assert lib.qoda_linear(linear(rows=0, x=0, y=0), None, 0, None) == qoda.OK
    assert lib.qoda_linear(linear(cout=0, w=0, y=0), None, 0, None) == qoda.OK
    for rows, cin, cout in ((0, 5, 7), (5, 0, 7), (5, 7, 0), (0, 0, 0)):
        assert lib.qoda_linear_workspace_bytes(linear(rows=rows, cin=cin, cout=cout, ys=8)) >= 0
        assert lib.qoda_linear_input_grad_workspace_bytes(ops._INPUT_GRAD.pack(0, 0, rows, cin, cout, 4096, 8, 4096, 8, 0, 8, 0, 8, 8192, 8, 0.0, 0, 0)) >= 0
        assert lib.qoda_linear_weight_grad_workspace_bytes(ops._WEIGHT_GRAD.pack(0, 0, rows, cin, cout, 4096, 8, 4096, 8, 8192, 8, 4096)) >= 0
    assert lib.qoda_dropout(ops._DROPOUT.pack(0, 0, 0, 8, 0, 0, 0, 0, 0, 0, 0.5, 0, 0), None) == qoda.OK
    assert lib.qoda_group_norm(ops._NORM.pack(0, 0, 0, 3, 8, 2, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 1e-5), None, 0, None) == qoda.OK


def test_an_error_belongs_to_its_thread(lib):
    import threading

    assert lib.qoda_linear(linear(dtype=9), None, 0, None) == qoda.EINVAL
    other = []
    t = threading.Thread(target=lambda: other.append(lib.qoda_operator_error()))
    t.start()
    t.join()
    assert other == [b""] and b"dtype 9" in lib.qoda_operator_error()


def test_definitions_generator_against_known_answers():
    """The generator that the expected masks come from, against the vectors that pin the quantizer's."""
    for line in open(os.path.join(ROOT, "tests", "golden", "philox4x32_10_kat.txt")):
        if line.startswith("#") or not line.strip():
            continue
        v = [int(s, 16) for s in line.split()]
        assert [int(w) for w in D.philox([np.uint64(c) for c in v[:4]], v[4:6])] == v[6:]


def test_share_of_kept_entries():
    n = 1 << 16
    for p in (0.1, 0.5, 0.9):
        share = (D.lots(64, n // 64, 7, 3) >= D.threshold(p)).mean()
        assert abs(share - (1 - p)) < 5 * np.sqrt(p * (1 - p) / n)
    assert (D.lots(64, 64, 7, 3) != D.lots(64, 64, 7, 4)).mean() > 0.99


@pytest.mark.parametrize("activation", [["gelu"], {}, None, 3])
def test_an_activation_of_another_type_is_refused_as_a_value(lib, activation):
    x = pytest.importorskip("torch").zeros((2, 2))
    s = x[:, 0]
    for call in (lambda: ops.linear(x, x, activation=activation), lambda: ops.linear_input_grad(x, x, pre=x, activation=activation),
                 lambda: ops.dropout(x, 0.5, 1, 1, activation=activation), lambda: ops.dropout_grad(x, 0.5, 1, 1, pre=x, activation=activation),
                 lambda: ops.group_norm(x, 1, activation=activation), lambda: ops.group_norm_grad(x, x, s, s, 1, activation=activation)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("positions,position,sample", [(1 << 30, 1 << 34, 24), ((1 << 31) - 65536, 1 << 33, 8), (1 << 30, 1 << 39, 1 << 49)])
def test_strides_whose_product_passes_64_bits_are_refused(lib, positions, position, sample):
    """Samples that would lie inside one another: what a sample spans is more than its stride, also where it is no 64-bit number."""
    dense = (8192, positions * 8, 8)
    for x, y in (((4096, sample, position), dense), (dense, (4096, sample, position))):
        a = ops._NORM.pack(0, 0, 2, positions, 8, 2, *x, *y, 0, 0, 4096, 4096, 1e-5)
        assert lib.qoda_group_norm_workspace_bytes(a) == qoda.EINVAL and b"strides" in lib.qoda_operator_error()
