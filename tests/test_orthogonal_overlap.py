"""Updates whose result would lie in some of g's entries without being g: refused (CPU).  Workgroups would overwrite what others still read."""
import os

import numpy as np
import pytest

from paper_2505_14371_amd import matrices as mats
from paper_2505_14371_amd import qoda

A = 1 << 20            # an address that is never followed


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(qoda.LIB_PATH):
        from paper_2505_14371_amd import build

        build.build()
    return mats._load()


def answer(lib, n, rows, cols, g, x, dtype=0):
    return lib.qoda_orthogonalize_workspace_bytes(mats._ORTHOGONALIZE.pack(dtype, 5, n, rows, cols, *g, *x, *mats.QUINTIC, 1e-7))


def entries(n, rows, cols, first, matrix, row):
    return {first + i * matrix + j * row + k for i in range(n) for j in range(rows) for k in range(cols)}


@pytest.mark.parametrize("alike", [True, False])
def test_as_the_entries_say(lib, alike):
    rng = np.random.default_rng(int(alike))
    seen = [0, 0]
    for _ in range(4000):
        n, rows, cols, dtype = (int(v) for v in rng.integers([1, 1, 1, 0], [4, 5, 6, 2]))
        strides = []
        for _ in range(2):
            row = cols + int(rng.integers(0, 2 * cols + 1))
            strides.append(((rows - 1) * row + cols + int(rng.integers(0, 12)), row))
        if alike:
            strides[1] = strides[0]
        off, size = int(rng.integers(-40, 41)), (4, 2)[dtype]
        g, x = (A, *strides[0]), (A + off * size, *strides[1])
        both = entries(n, rows, cols, 0, *strides[0]) & entries(n, rows, cols, off, *strides[1])
        itself = off == 0 and (strides[0][0] == strides[1][0] or n == 1) and (strides[0][1] == strides[1][1] or rows == 1)
        got = answer(lib, n, rows, cols, g, x, dtype)
        assert (got >= 0) == (itself or not both), (n, rows, cols, off, strides, got)
        if got < 0:
            assert "neither g nor apart" in lib.qoda_operator_error().decode()
        seen[int(got >= 0)] += 1
    assert min(seen) > 500


def test_columns_of_one_buffer_and_far_ones(lib):
    rows, cols = 1 << 16, 1 << 10
    assert answer(lib, 1, rows, cols, (A, 0, 2 * cols), (A + 4 * cols, 0, 2 * cols)) >= 0               # left and right half of rows
    assert answer(lib, 1, rows, cols, (A, 0, 2 * cols), (A + 4 * cols - 4, 0, 2 * cols)) == qoda.EINVAL
    assert answer(lib, 40, 1000, cols, (A, 10**6 * 3, 1500), (A + 4 * (1500 * 999 + cols), 10**6 * 3, 1500)) >= 0      # between the matrices
    far = 1 << 45
    assert answer(lib, 2, rows, cols, (A, 1 << 40, cols), (A + far, 1 << 40, cols)) >= 0
    assert answer(lib, 2, rows, cols, (A + (4 << 40), 1 << 40, cols), (A, 1 << 40, cols)) == qoda.EINVAL  # x's second matrix is g's first
