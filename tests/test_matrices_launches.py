"""What the calls of include/qoda_matrices.h would launch, seen on the CPU: the host side over stand-ins for the HIP runtime
(tests/matrices_launch_stand_in.cpp).  HIP launches fewer than 2^32 work-items along a dimension of the grid, so sizes that the header accepts may take
several launches."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

from paper_2505_14371_amd import build
from paper_2505_14371_amd import matrices as mats

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2505_14371_amd", "csrc")
SIDE = 0x7FFF0000
ceil = lambda a, b: -(-a // b)  # noqa: E731
A = 4096


@pytest.fixture(scope="session")
def lib(tmp_path_factory):
    hipcc, gxx = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), shutil.which("g++")
    if not os.path.exists(hipcc) or gxx is None or shutil.which("nm") is None:
        pytest.skip("no hipcc, g++ or nm")
    d = tmp_path_factory.mktemp("launches")
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-Wall", "-O3")]
    objects = []
    for src in [os.path.join(CSRC, f) for f in ("qoda_mx_quantize.hip", "qoda_mx_product.hip", "qoda_orthogonal.hip", "qoda_matrices_api.hip")] + [
            os.path.join(HERE, "matrices_launch_stand_in.cpp")]:
        objects.append(str(d / (os.path.basename(src) + ".o")))
        done = subprocess.run([hipcc, *flags, "-O1", "-w", "--offload-host-only", "-x", "hip", "-c", src, "-o", objects[-1]], capture_output=True, text=True)
        assert done.returncode == 0, done.stderr[-4000:]
    # there is no device code: the places where the launches' object files expect it are not looked at
    nowhere = sorted(set(re.findall(r"U (__hip_fatbin\w*)", subprocess.run(["nm", "-u", *objects], capture_output=True, text=True, check=True).stdout)))
    so = str(d / "liblaunches.so")
    done = subprocess.run([gxx, "-shared", "-Wl,-Bsymbolic", *[f"-Wl,--defsym={n}=0" for n in nowhere], *objects, "-o", so], capture_output=True, text=True)
    assert done.returncode == 0, done.stderr[-4000:]
    L = ctypes.CDLL(so)
    for name in ("mx_linear", "mx_linear_input_grad", "mx_linear_weight_grad", "orthogonalize"):
        size, call = getattr(L, f"qoda_{name}_workspace_bytes"), getattr(L, f"qoda_{name}")
        size.argtypes, size.restype = [ctypes.c_char_p], ctypes.c_int64
        call.argtypes, call.restype = [ctypes.c_char_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p], ctypes.c_int
    for call in (L.qoda_mx_quantize, L.qoda_mx_values):
        call.argtypes, call.restype = [ctypes.c_char_p, ctypes.c_void_p], ctypes.c_int
    L.stand_in_log.restype, L.qoda_operator_error.restype = ctypes.c_char_p, ctypes.c_char_p
    return L


def launches(lib, name, args):
    """[(kernel, workgroups of all its launches one after the other, number of these)] of a call, each launch looked at."""
    lib.stand_in_reset()
    if name in ("mx_quantize", "mx_values"):
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


def quantize(rows, cols, transposed=0, stochastic=0, dtype=1):
    return mats._QUANTIZE.pack(dtype, transposed, stochastic, rows, cols, A, cols, A, A, 0, 0)


def linear(rows, cin, cout, plain=True, dtype=1):
    return mats._LINEAR.pack(dtype, 0, rows, cin, cout, *((A, cin, 0, 0) if plain else (0, 0, A, A)), A, A, 0, 0, A, cout, 0, 0, 0, 0.0, 0, 0)


def weight_grad(rows, cin, cout, bias=A):
    return mats._WEIGHT_GRAD.pack(0, rows, cin, cout, A, A, A, A, A, cin, bias)


def orthogonalize(n, rows, cols, steps=1, dtype=0):
    return mats._ORTHOGONALIZE.pack(dtype, steps, n, rows, cols, A, rows * cols, cols, A, rows * cols, cols, *mats.QUINTIC, 1e-7)


@pytest.mark.parametrize("rows,cols", [(1 << 20, 1 << 19), (SIDE, 40), (40, SIDE), (1000, 300)])
@pytest.mark.parametrize("transposed", [0, 1])
def test_rounding_and_values(lib, rows, cols, transposed):
    many = ceil(rows, 64) * ceil(cols, 256) if not transposed else ceil(cols, 64) * ceil(rows, 256)
    (kernel, workgroups, pieces), = launches(lib, "mx_quantize", quantize(rows, cols, transposed))
    assert kernel.startswith("k_mx_columns" if transposed else "k_mx_rows") and workgroups == many and (pieces > 1) == (many >= 1 << 24)
    if not transposed:
        (kernel, workgroups, pieces), = launches(lib, "mx_values", mats._VALUES.pack(0, rows, cols, A, A, A, cols))
        assert kernel == "k_mx_values<float>" and workgroups == many


def test_products(lib):
    short = lambda got: [k[0].split("<")[0] for k in got]  # noqa: E731
    assert short(launches(lib, "mx_linear", linear(1, 2048, 8192))) == ["k_mx_few_rows"]                      # one launch, rounding in it
    assert short(launches(lib, "mx_linear", linear(1, 8192, 50304))) == ["k_mx_rows", "k_mx_few_rows"]
    assert short(launches(lib, "mx_linear", linear(1, 8192, 50304, plain=False))) == ["k_mx_few_rows"]
    assert short(launches(lib, "mx_linear", linear(3300, 410, 2100))) == ["k_mx_rows", "k_mx_product"]
    assert short(launches(lib, "mx_linear", linear(33, 8192, 2048, plain=False))) == ["k_mx_product", "k_join"]
    assert short(launches(lib, "mx_linear_weight_grad", weight_grad(100000, 64, 64))) == ["k_mx_product", "k_join"]
    assert short(launches(lib, "mx_linear_weight_grad", weight_grad(100000, 64, 64, bias=0))) == ["k_mx_product", "k_join"]
    assert short(launches(lib, "mx_linear_weight_grad", weight_grad(0, 64, 64))) == ["k_mx_product"]      # zeros
    def tiles_and_sums(rows, cin, cout, bias):
        (kernel, workgroups, _), *_ = launches(lib, "mx_linear_weight_grad", weight_grad(rows, cin, cout, bias))
        side, *_, wm, wn = map(int, re.match(r"k_mx_product<float,2,(\d+),(\d+),(\d+),(\d+)>", kernel).groups())
        tiles = ceil(cout, side) * ceil(cin, side)
        return workgroups - tiles, ceil(cout, wm * wn)
    assert tiles_and_sums(300, 410, 2100, 0)[0] == 0
    for sizes in ((300, 410, 2100), (0, 64, 70), (8192, 2048, 6144), (100, 0, 70)):      # sums of rows by workgroups behind the tiles', a row a wave
        sums, rows = tiles_and_sums(*sizes, A)
        assert sums == rows
    sums, rows = tiles_and_sums(100000, 64, 64, A)                                         # ... of all the parts
    assert 0 < sums < rows
    assert launches(lib, "mx_linear_weight_grad", weight_grad(100, 0, 70, 0)) == launches(lib, "mx_linear_weight_grad", weight_grad(100, 70, 0)) == []
    assert launches(lib, "mx_linear", linear(5, 8, 0)) == launches(lib, "mx_linear", linear(0, 8, 5)) == []
    (kernel, workgroups, pieces), = launches(lib, "mx_linear", linear(1, 1, SIDE, plain=False))
    assert kernel.startswith("k_mx_few_rows<") and workgroups == ceil(SIDE, 32) and pieces > 1
    kernel, workgroups, pieces = launches(lib, "mx_linear", linear(SIDE, 1, 1, plain=False))[0]
    side = int(re.match(r"k_mx_product<\w+,0,(\d+),", kernel).group(1))
    assert workgroups == ceil(SIDE, side) and pieces > 1
    sums, rows = tiles_and_sums(1, 1, SIDE, A)
    assert sums == rows


def test_orthogonalisation(lib):
    short = lambda got: [k[0].split("<")[0] for k in got]  # noqa: E731
    assert launches(lib, "orthogonalize", orthogonalize(3, 40, 50, steps=5)) == [("k_small<float,1,81792>", 3, 1)]
    assert launches(lib, "orthogonalize", orthogonalize((1 << 23) + 5, 4, 5, steps=5)) == [("k_small<float,1,40832>", (1 << 23) + 5, 2)]
    assert short(launches(lib, "orthogonalize", orthogonalize(3, 400, 500, steps=0))) == ["k_squares", "k_start"]
    got = short(launches(lib, "orthogonalize", orthogonalize(1, 400, 500, steps=2)))
    assert [k for k in got if k != "k_pair_join"] == ["k_squares", "k_start"] + ["k_pair_product"] * 6
    got = launches(lib, "orthogonalize", orthogonalize(1 << 17, 300, 300))
    assert got[1][:2] == ("k_start<float,true>", (1 << 17) * 25) and got[-1][2] > 0
    got = launches(lib, "orthogonalize", orthogonalize(1 << 21, 300, 300))
    side = int(re.match(r"k_pair_product<(\d+),", got[2][0]).group(1))
    t = ceil(320, side)
    assert got[2][1] == (1 << 21) * t * (t + 1) // 2 and got[1][2] > 1


def split_products(lib, *sizes):
    """[(side of the tiles, side of the join's tiles, whether the product is symmetric)] of an update's products whose sums are split."""
    got, out = launches(lib, "orthogonalize", orthogonalize(*sizes)), []
    n, rows, cols = sizes[:3]
    m = ceil(min(rows, cols), 32) * 32
    for (kernel, workgroups, _), (join, joins, _) in zip(got, got[1:]):
        if join.startswith("k_pair_join"):
            side = int(re.match(r"k_pair_product<(\d+),", kernel).group(1))
            of_join = int((re.search(r"<(\d+)>", join) or [0, 64])[1])
            t, tj = ceil(m, side), ceil(m, of_join)
            symmetric = workgroups == n * t * (t + 1) // 2
            assert not symmetric or joins == n * tj * (tj + 1) // 2
            out.append((side, of_join, symmetric))
    return out


# a batch's smaller side times the larger one, of which several take tiles of 96 with their sums in parts
@pytest.mark.parametrize("sizes", [(3, 672, 4000), (1, 1440, 2176), (8, 480, 2048), (16, 288, 1500), (2, 544, 9000), (4, 576, 3100), (1, 672, 30000), (21, 288, 1200), (1, 2048, 8192), (1, 1000, 1000)])
def test_a_join_takes_no_entry_of_a_symmetric_product_that_was_not_computed(lib, sizes):
    """Of a symmetric product the tiles with row <= column are computed, and of the join's tiles those are finished whole: each has to lie in one of the product's."""
    for side, of_join, symmetric in split_products(lib, *sizes):
        assert not symmetric or side % of_join == 0, (side, of_join)


def test_tiles_of_96_are_split(lib):
    """That the sizes above reach them."""
    for sizes in ((3, 672, 4000), (1, 1440, 2176)):
        assert (96, 32, True) in split_products(lib, *sizes)


def test_orthogonalisation_by_norm(lib):
    """Polynomials whose bound may be far above the singular values: norms of X and A in every step, whatever the size; a join of every product that has a matrix's own factors."""
    step = ["k_squares<float>", "k_start<float,true>", "k_pair_product", "k_squares<float>", "k_start<float,true>", "k_start_scales", "k_pair_product", "k_pair_join", "k_pair_product", "k_pair_join"]
    for n, rows, cols, dtype in ((3, 20, 30, 0), (1, 61, 37, 1), (40, 300, 410, 0)):
        for co in ((0.0, 1.0, 0.0), (0.9, 0.9, 0.9), (1e-30, 1e-30, 0.0)):
            args = mats._ORTHOGONALIZE.pack(dtype, 2, n, rows, cols, A, rows * cols, cols, A, rows * cols, cols, *co, 1e-7)
            got = [k if k.startswith("k_s") else k.split("<")[0] for k, _, _ in launches(lib, "orthogonalize", args)]
            first = [k.replace("float", "bf16") if dtype and at < 2 else k for at, k in enumerate(step)]
            assert got == first + step, got
    for co, steps in ((mats.QUINTIC, 5), (mats.QUINTIC, 1000), ((1.5, -0.5, 0.0), 100), ((2.0, -1.5, 0.5), 30), ((1.875, -1.25, 0.375), 30), ((1.0, 0.0, 0.0), 4), ((4.0848, -6.8946, 2.9270), 5)):
        args = mats._ORTHOGONALIZE.pack(0, steps, 1, 300, 410, A, 0, 410, A, 0, 410, *co, 1e-7)          # the usual ones are not
        assert "k_start_scales" not in [k for k, _, _ in launches(lib, "orthogonalize", args)], co
