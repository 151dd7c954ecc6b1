"""What the operators' calls would launch, seen on the CPU: the host side over stand-ins for the HIP runtime (tests/operators_launch_stand_in.cpp).
HIP launches fewer than 2^32 work-items along a dimension of the grid, so sizes that the header accepts may take several launches."""
import ctypes
import math
import os
import re
import shutil
import subprocess

import pytest

from paper_2505_14371_amd import build
from paper_2505_14371_amd import operators as ops

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2505_14371_amd", "csrc")
SIDE = 0x7FFF0000


@pytest.fixture(scope="session")
def lib(tmp_path_factory):
    hipcc, gxx = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), shutil.which("g++")
    if not os.path.exists(hipcc) or gxx is None or shutil.which("nm") is None:
        pytest.skip("no hipcc, g++ or nm")
    d = tmp_path_factory.mktemp("launches")
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-Wall", "-O3")]
    objects = []
    for src in [os.path.join(CSRC, f) for f in ("qoda_linear.hip", "qoda_dropout.hip", "qoda_group_norm.hip", "qoda_operators_api.hip")] + [
            os.path.join(HERE, "operators_launch_stand_in.cpp")]:
        objects.append(str(d / (os.path.basename(src) + ".o")))
        done = subprocess.run([hipcc, *flags, "-O1", "-w", "--offload-host-only", "-x", "hip", "-c", src, "-o", objects[-1]], capture_output=True, text=True)
        assert done.returncode == 0, done.stderr[-4000:]
    # there is no device code: the places where the launches' object files expect it are not looked at
    nowhere = sorted(set(re.findall(r"U (__hip_fatbin\w*)", subprocess.run(["nm", "-u", *objects], capture_output=True, text=True, check=True).stdout)))
    so = str(d / "liblaunches.so")
    done = subprocess.run([gxx, "-shared", "-Wl,-Bsymbolic", *[f"-Wl,--defsym={n}=0" for n in nowhere], *objects, "-o", so], capture_output=True, text=True)
    assert done.returncode == 0, done.stderr[-4000:]
    L = ctypes.CDLL(so)
    for name in ("linear", "linear_input_grad", "linear_weight_grad", "group_norm", "group_norm_grad"):
        size, call = getattr(L, f"qoda_{name}_workspace_bytes"), getattr(L, f"qoda_{name}")
        size.argtypes, size.restype = [ctypes.c_char_p], ctypes.c_int64
        call.argtypes, call.restype = [ctypes.c_char_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p], ctypes.c_int
    for call in (L.qoda_dropout, L.qoda_dropout_grad):
        call.argtypes, call.restype = [ctypes.c_char_p, ctypes.c_void_p], ctypes.c_int
    L.stand_in_log.restype, L.qoda_operator_error.restype = ctypes.c_char_p, ctypes.c_char_p
    return L


def launches(lib, name, args):
    """[(kernel, workgroups of all its launches one after the other, number of these)] of a call, each launch looked at."""
    lib.stand_in_reset()
    if name.startswith("dropout"):
        assert getattr(lib, "qoda_" + name)(args, None) == 0, lib.qoda_operator_error()
    else:
        need = getattr(lib, f"qoda_{name}_workspace_bytes")(args)
        assert need >= 0, lib.qoda_operator_error()
        assert getattr(lib, "qoda_" + name)(args, 1 << 20 if need else None, need, None) == 0, lib.qoda_operator_error()
    out = []
    for line in lib.stand_in_log().decode().splitlines():
        kernel, x, y, z, threads, first = line.rsplit(" ", 5)
        x, y, z, threads, first = int(x), int(y), int(z), int(threads), int(first)
        assert 0 < x * threads < 1 << 32 and 0 < y < 65536 and z == 1, line
        if first == 0:
            out.append([kernel, 0, 0])
        assert out[-1][0] == kernel and out[-1][1] == first, line           # goes on where the launch before it ended
        out[-1][1] += x
        out[-1][2] += 1
    return [tuple(v) for v in out]


ceil = lambda a, b: -(-a // b)  # noqa: E731
at = lambda stride: (4096, stride)  # noqa: E731


def linear(rows, cin, cout, dtype=1):
    return ops._LINEAR.pack(dtype, 0, rows, cin, cout, *at(cin), *at(cin), 0, 0, *at(cout), 0, 0, 0, 0.0, 0, 0)


def norm(n, s, c, groups, dtype=1):
    three = (4096, s * c, c)
    return ops._NORM.pack(dtype, 0, n, s, c, groups, *three, *three, 0, 0, 4096, 4096, 1e-5)


def norm_grad(n, s, c, groups, dtype=1, sums=4096):
    three = (4096, s * c, c)
    return ops._NORM_GRAD.pack(dtype, 0, n, s, c, groups, *three, *three, 0, 0, 0, *three, 0, 0, 4096, 4096, sums, sums, 0)


# rows of one eight a lane in teams of 16 and 64, of four, in a workgroup each, and longer: rows, channels, workgroup's rows
ROWS = [((1 << 28) + 5, 8, 16), ((1 << 26) + 5, 136, 4), ((1 << 26) + 5, 520, 4), ((1 << 24) + 5, 2056, 1), ((1 << 22) + 5, 8200, 1), (1000, 8, 16)]


@pytest.mark.parametrize("rows,channels,each", ROWS)
def test_rows_of_a_norm(lib, rows, channels, each):
    (kernel, workgroups, pieces), = launches(lib, "group_norm", norm(rows, 1, channels, 1))
    assert workgroups == ceil(rows, each) and (pieces > 1) == (rows > 1000), kernel
    names = [k[0].split("<")[0] for k in launches(lib, "group_norm_grad", norm_grad(rows, 1, channels, 1))]
    assert names == (["k_norm_long_channels", "k_norm_long_rows_grad"] if channels > 8192 else ["k_norm_rows_grad"]) + ["k_norm_join"]


@pytest.mark.parametrize("groups,len", [((1 << 24) + 5, 2), ((1 << 24) + 5, 40), (1 << 26, 16)])
def test_many_groups_of_a_row(lib, groups, len):
    """The gradient's workgroups are those of a group; dweight and dbias have 16 columns a workgroup."""
    got = launches(lib, "group_norm_grad", norm_grad(1, 1, groups * len, groups))
    assert got[0][:2] == (got[0][0], groups) and got[0][0].startswith("k_norm_rows_grad<") and got[0][2] > 1
    assert got[1][:2] == ("k_norm_join", ceil(2 * groups * len, 16)) and got[1][2] > 1 and got[2:] == []


def test_maps_in_waves(lib):
    n = (1 << 26) + 3
    (kernel, workgroups, pieces), = launches(lib, "group_norm", norm(n, 2, 1, 1))
    assert kernel.startswith("k_norm_maps<") and workgroups == n and pieces == 2
    got = launches(lib, "group_norm_grad", norm_grad(n, 2, 1, 1))
    assert got[0][1:] == (n, 2) and got[0][0].startswith("k_norm_maps_grad<") and [k[:1] for k in got[1:]] == [("k_norm_join",)] * 2


def test_maps_in_pieces(lib):
    """Statistics and sums joined by workgroups of 1024: of 2^22 groups and more."""
    short = lambda got: [k[0].split("<")[0] for k in got]  # noqa: E731
    got = launches(lib, "group_norm", norm(33000, 300000, 128, 128, dtype=0))
    assert short(got) == ["k_norm_maps", "k_norm_maps_join", "k_norm_maps"] and got[1][1] == 33000 * 128 and got[1][2] == 2
    assert short(launches(lib, "group_norm", norm(40, 1000, 64, 2))) == ["k_norm_maps"]
    assert short(launches(lib, "group_norm", norm(40, 5000, 64, 2))) == ["k_norm_maps"] * 2
    n = (1 << 22) + 3
    got = launches(lib, "group_norm_grad", norm_grad(n, 2, 4100, 1))
    assert short(got) == ["k_norm_maps_grad", "k_norm_join", "k_norm_group_sums", "k_norm_maps_grad", "k_norm_join", "k_norm_join"]
    assert got[1][1] == n * ceil(2 * 4100, 16) and got[2][1] == n and got[1][2] > 1 and got[2][2] > 1
    assert short(launches(lib, "group_norm_grad", norm_grad(40, 4000, 64, 2))) == ["k_norm_maps_grad", "k_norm_maps_grad", "k_norm_join"]


def test_products(lib):
    """One row by many; many rows by one; the largest sides."""
    (kernel, workgroups, pieces), = launches(lib, "linear", linear(1, 1, (1 << 28) + 40))
    assert kernel.startswith("k_few_rows<") and workgroups == ceil((1 << 28) + 40, 16) and pieces == 2
    for rows in ((1 << 30) + 100, SIDE):
        (kernel, workgroups, pieces), = launches(lib, "linear", linear(rows, 1, 1))
        tile = int(re.match(r"k_product<\w+,0,(\d+),", kernel).group(1))
        assert workgroups == ceil(rows, tile) and pieces == ceil(workgroups, ((1 << 32) - 1) // 256)
    for cin, cout in ((SIDE, 1), (1, SIDE)):
        assert launches(lib, "linear", linear(1, cin, cout))
        assert launches(lib, "linear_weight_grad", ops._WEIGHT_GRAD.pack(1, 0, 1, cin, cout, *at(cout), *at(cin), *at(cin), 4096))
        assert launches(lib, "linear_input_grad", ops._INPUT_GRAD.pack(1, 0, 1, cin, cout, *at(cout), *at(cin), 0, 0, 0, 0, *at(cin), 0.0, 0, 0))


@pytest.mark.parametrize("rows,cols", [(SIDE, 64), (SIDE, 57), (1 << 20, 1 << 17), (1, SIDE), (SIDE, 1)])
def test_entries(lib, rows, cols):
    args = ops._DROPOUT.pack(1, 0, rows, cols, *at(cols), 0, 0, *at(cols), 0.5, 0, 0)
    (kernel, workgroups, pieces), = launches(lib, "dropout", args)
    assert workgroups == ceil(rows * ceil(cols, 8), 1024) and pieces == math.ceil(workgroups * 256 / ((1 << 32) - 256))
