"""The bound on singular values that an update's polynomial is refused by (CPU), against the polynomial's values on a grid."""
import os

import numpy as np
import pytest

from paper_2505_14371_amd import matrices as mats
from paper_2505_14371_amd import qoda

A = 4096            # an address that is never followed


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(qoda.LIB_PATH):
        from paper_2505_14371_amd import build

        build.build()
    return mats._load()


def taken(lib, coefficients, steps):
    args = mats._ORTHOGONALIZE.pack(0, steps, 1, 300, 400, A, 0, 400, A, 0, 400, *coefficients, 1e-7)
    need = lib.qoda_orthogonalize_workspace_bytes(args)
    assert need > 0 or (need == qoda.EINVAL and "2^40" in lib.qoda_operator_error().decode())
    return need > 0


def greatest(coefficients, steps):
    """The largest of the bounds on |X| and on |b A + c A A| of all steps, from values on a grid (less than they are by its spacing's square)."""
    a, b, c = coefficients
    top, seen = 1.0, 0.0
    for _ in range(steps):
        s = np.linspace(0, top, 20001)
        seen = max(seen, np.abs(b * s**2 + c * s**4).max())
        top = np.abs(a * s + b * s**3 + c * s**5).max()
        seen = max(seen, top)
        if seen > 2.0**60:
            break
    return seen


# a root of the slope by the difference of two numbers that are nearly the same is lost for these c, and with it the largest value
TINY = [0.0, 1e-17, -1e-17, 5.5e-17, 1e-12, -1e-9, 1e-300, 5e-324, -1e-310]


@pytest.mark.parametrize("c", TINY)
def test_a_last_coefficient_next_to_nothing(lib, c):
    assert not taken(lib, (6.0, -6.0, c), 6)            # 2.3, 60, 1.3e6, 1e19
    assert taken(lib, (6.0, -6.0, c), 3)
    assert taken(lib, (2.0, -2.0, c), 1000)             # 0.77, 0.77, ...
    assert not taken(lib, (-6.0, 6.0, c), 6)


def test_polynomials_of_all_kinds(lib):
    rng = np.random.default_rng(5)
    seen = [0, 0]
    for k in range(700):
        a, b, c = rng.choice([-1.0, 1.0], 3) * 10.0 ** rng.uniform([-3, -3, -18], [2, 2, 2])
        if k % 7 == 0:
            b = 0.0
        if k % 11 == 0:
            a = 0.0
        steps = int(rng.integers(1, 9))
        v = greatest((a, b, c), steps)
        if not 2.0**39.9 < v < 2.0**40.1:               # nearer to the border than the grid is sure of
            assert taken(lib, (a, b, c), steps) == (v < 2.0**40), (a, b, c, steps, v)
            seen[int(v < 2.0**40)] += 1
    assert min(seen) > 70, seen


def test_polynomials_that_the_gpu_tests_take(lib):
    for co, steps in (((1.0, 10.0, 80.0), 2), ((0.9, 0.9, 0.9), 3), ((1.0, 1.0, 0.5), 3), ((0.0, 1.0, 0.0), 3), ((0.0, 0.0, 1.0), 2), ((0.5, 0.5, 0.0), 60), ((1e-30, 1e-30, 0.0), 1)):
        assert taken(lib, co, steps), co
    assert not taken(lib, (1.0, 1.0, 1.0), 3) and not taken(lib, (1.0, 100.0, 1000.0), 2)
