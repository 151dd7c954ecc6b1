"""Updates by polynomials other than the usual ones, against the formula in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import matrix_definitions as M  # noqa: E402
from paper_2505_14371_amd import matrices as mats  # noqa: E402
from test_gpu_orthogonal import check, matrices, put  # noqa: E402


@pytest.fixture(autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("a GPU test was selected but no GPU is visible")


@pytest.mark.parametrize("shape", [(37, 61), (130, 200), (300, 70)])
@pytest.mark.parametrize("c", [5.5e-17, -1e-17, 1e-300])
@pytest.mark.parametrize("steps", [2, 5])
def test_a_last_coefficient_next_to_nothing(shape, c, steps):
    """What c = 0 gives, with the bound that numbers are scaled by."""
    g, gd = put(matrices(np.random.default_rng(shape), 2, *shape), "f32")
    x = mats.orthogonalize(g, steps=steps, coefficients=(2.0, -2.0, c))
    check(x, gd, steps, (2.0, -2.0, c), 1e-7, "f32")
    assert torch.equal(x, mats.orthogonalize(g, steps=steps, coefficients=(2.0, -2.0, 0.0)))


def off_by(sv, steps, coefficients, m, k):
    """Of the Frobenius norm of the error, from the singular values that X_0 has, not from a bound on them.  A step takes a X, A = X X^T, B = b A + c A A and B X: a pair holds 2^-22 of
    a number, a sum of k terms in fp32 is off by 2^-24 root(k) of what it adds up, and of B no more is lost than 2^-41 of |b||A| + |c||A|^2 in each entry.  What is off is multiplied by
    the largest slope in each later step."""
    a, b, c = coefficients
    unit, off = 2.0**-22 + np.sqrt(k) * 2.0**-24, 2.0**-22 * np.linalg.norm(sv)
    for _ in range(steps):
        top, norm, square = np.abs(sv).max(), np.linalg.norm(sv), np.linalg.norm(sv**2)
        s = np.linspace(0, top, 4001)
        off = off * np.abs(a + 3 * b * s**2 + 5 * c * s**4).max()
        off += 4 * unit * (abs(a) + abs(b) * top**2 + abs(c) * top**4) * norm + m * 2.0**-41 * (abs(b) * square + abs(c) * square**2) * norm
        sv = a * sv + b * sv**3 + c * sv**5
    return off


# small singular values fall, or large ones grow faster than small ones
FAR = [((0.0, 1.0, 0.0), 3), ((0.0, 0.0, 1.0), 2), ((1.0, 10.0, 80.0), 2), ((0.9, 0.9, 0.9), 3), ((1.0, 1.0, 0.5), 3), ((0.5, 0.5, 0.0), 60), ((1e-30, 1e-30, 0.0), 1), ((1e-3, 1e-4, 1e-4), 7),
       ((100.0, -20.0, 3.0), 2), ((0.0, 1e-3, 10.0), 2), ((-0.01, 0.02, -2.0), 3), ((3.0, 1.0, 0.0), 3)]


@pytest.mark.parametrize("coefficients,steps", FAR)
@pytest.mark.parametrize("m,n,flat", [(5, 3, False), (37, 61, False), (61, 37, True), (130, 200, True), (300, 70, False), (500, 700, True)])
def test_singular_values_far_below_the_bound(coefficients, steps, m, n, flat):
    """As accurate as they are: digits are not lost to a bound that no singular value comes near."""
    rng = np.random.default_rng([m, n])
    a = rng.standard_normal((2, m, n))
    if flat:                                            # all singular values alike
        u, _, v = np.linalg.svd(a, full_matrices=False)
        a = u @ v
    g, gd = put(a * 1e-3, "f32", pad=3)
    got = mats.orthogonalize(g, steps=steps, coefficients=coefficients)
    assert torch.equal(mats.orthogonalize(g, steps=steps, coefficients=coefficients), got)
    want = M.orthogonalize(gd, steps, coefficients, 1e-7)
    for q, w, x in zip(got.double().cpu().numpy(), want, gd):
        sv = np.linalg.svd(x / (np.linalg.norm(x) + 1e-7), compute_uv=False)
        b = off_by(sv, steps, coefficients, min(m, n), max(m, n))
        off, size = np.linalg.norm(q - w), np.linalg.norm(w)
        assert off <= b + 2.0**-24 * size + 1e-44 * np.sqrt(w.size), (off, b, size)
    assert mats.orthogonalize(g, steps=steps, coefficients=coefficients, out=g) is g and torch.equal(g, got)


def test_by_norm_in_bf16_and_many():
    gen = torch.Generator("cuda").manual_seed(3)
    co = (0.5, 0.7, 0.9)
    g = torch.randn((70, 40, 50), device="cuda", generator=gen).bfloat16()
    x = mats.orthogonalize(g, steps=3, coefficients=co)
    wide = mats.orthogonalize(g.float(), steps=3, coefficients=co)
    assert torch.equal(x, wide.bfloat16())
    for k in (0, 33, 69):
        assert torch.equal(mats.orthogonalize(g[k], steps=3, coefficients=co), x[k])


@pytest.mark.parametrize("shape", [(3, 40, 50), (2, 300, 200)])
def test_by_norm_nothing_zeros_and_nan(shape):
    co = (0.5, 0.5, 0.25)
    g = torch.randn(shape, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    want = mats.orthogonalize(g, steps=4, coefficients=co)
    g[1] = 0.0
    x = mats.orthogonalize(g, steps=4, coefficients=co)
    assert torch.equal(x[0], want[0]) and torch.equal(x[1], torch.zeros_like(x[1]))
    assert torch.isnan(mats.orthogonalize(g, steps=4, coefficients=co, eps=0.0)[1]).all()
    for bad in (float("inf"), float("nan")):
        g[1, 3, 5] = bad
        x = mats.orthogonalize(g, steps=4, coefficients=co)
        assert torch.isnan(x[1]).all() and torch.equal(x[0], want[0])
    assert mats.orthogonalize(g[:0], steps=4, coefficients=co).shape == (0, *shape[1:])


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e30])
def test_by_norm_any_magnitude(scale):
    """Also where eps is far above g."""
    g, gd = put(matrices(np.random.default_rng(4), 40, 50) * scale, "f32")
    co, steps = (0.1, 1.0, 0.25), 2
    for eps in (0.0, 1e-7):
        x = mats.orthogonalize(g, steps=steps, coefficients=co, eps=eps).double().cpu().numpy()
        w = M.orthogonalize(gd, steps, co, eps)
        sv = np.linalg.svd(gd / (np.linalg.norm(gd) + eps), compute_uv=False)
        assert np.linalg.norm(x - w) <= off_by(sv, steps, co, 40, 50) + 2.0**-24 * np.linalg.norm(w) + 1e-44 * np.sqrt(w.size)


def test_by_norm_captured_and_over_nan():
    """Replayed on new matrices; and through the C interface in a workspace of NaN."""
    co, steps = (0.5, 0.7, 0.9), 3
    gen = torch.Generator("cuda").manual_seed(9)
    g, out = torch.randn((3, 200, 310), device="cuda", generator=gen), torch.empty((3, 200, 310), device="cuda")
    mats.orthogonalize(g, steps=steps, coefficients=co, out=out)
    args = mats._ORTHOGONALIZE.pack(0, steps, 3, 200, 310, g.data_ptr(), 62000, 310, out.data_ptr(), 62000, 310, *co, 1e-7)
    lib = mats._load()
    need = lib.qoda_orthogonalize_workspace_bytes(args)
    work, want = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda"), out.clone()
    out.zero_()
    assert lib.qoda_orthogonalize(args, work.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(out, want) and (work[need:] == 255).all()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mats.orthogonalize(g, steps=steps, coefficients=co, out=out)
    for _ in range(3):
        g.copy_(torch.randn((3, 200, 310), device="cuda", generator=gen))
        want = mats.orthogonalize(g, steps=steps, coefficients=co)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
