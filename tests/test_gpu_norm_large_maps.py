"""Normalisations of maps that are cut into many pieces: their values, and a time that grows with the map, not with its square."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import operator_definitions as D  # noqa: E402
from paper_2505_14371_amd import operators as ops  # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("a GPU test was selected but no GPU is visible")


def milliseconds(work, turns=4):
    work()
    times = []
    for _ in range(turns):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        work()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b))
    return min(times)


# one group, many channels: pieces of few positions; many positions; a group wider than a block
@pytest.mark.parametrize("n,s,c,groups", [(1, 32768, 1024, 1), (1, 1 << 20, 64, 32), (1, 4096, 8192, 1)])
@pytest.mark.parametrize("gradient", [False, True])
def test_time_of_a_large_map(n, s, c, groups, gradient):
    """At most ten times a copy of what it reads and writes (a pass reads the map twice; it was up to hundreds of times)."""
    x = torch.randn((n, s, c), device="cuda").to(torch.bfloat16)
    y, mean, rstd = ops.group_norm(x, groups)
    to = torch.empty_like(x)
    copy = milliseconds(lambda: to.copy_(x))
    if gradient:
        assert milliseconds(lambda: ops.group_norm_grad(y, x, mean, rstd, groups)) <= 10 * 1.5 * copy + 0.1
    else:
        assert milliseconds(lambda: ops.group_norm(x, groups)) <= 10 * copy + 0.1


# pieces joined by a launch of their own, forward and backward; groups wider than a block and narrower, several samples, odd widths
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,s,c,groups", [(2, 40000, 64, 4), (1, 70000, 26, 2), (3, 1100, 1024, 1), (2, 700, 4100, 1), (1, 1300, 6000, 2), (1, 9, 70000, 7)])
def test_values_of_large_maps(n, s, c, groups, dtype):
    """Against the definition in 64 bits.  No sum has more than 600 additions one after the other (a thread's, a workgroup's rows, the pieces
    of a team, the lanes), so a mean of terms is off by at most 600 half units of the mean of their magnitudes."""
    gen = torch.Generator(device="cuda").manual_seed(s)
    draw = lambda *shape: torch.randn(shape, device="cuda", generator=gen)  # noqa: E731
    x, dy = ((0.5 + draw(n, s, c)).to(TYPES[dtype]), draw(n, s, c).to(TYPES[dtype]))
    w, b = 1 + 0.2 * draw(c), 0.2 * draw(c)
    y, mean, rstd = ops.group_norm(x, groups, w, b, activation="silu")
    dx, dw, db = ops.group_norm_grad(dy, x, mean, rstd, groups, w, b, activation="silu", residual=dy)
    unit, store = 600 * D.U32, D.STORE[dtype] * 1.001
    four = lambda t: t.double().view(n, s, groups, c // groups)  # noqa: E731
    X, W, B = four(x), w.double().view(groups, -1), b.double().view(groups, -1)
    m = X.mean((1, 3), keepdim=True)
    r = ((X - m).square().mean((1, 3), keepdim=True) + 1e-5).rsqrt()
    assert ((mean.double() - m.view(n, groups)).abs() <= unit * X.abs().mean((1, 3))).all()
    assert ((rstd.double() / r.view(n, groups) - 1).abs() <= unit).all()
    h = (X - m) * r
    z = h * W + B
    sig = torch.sigmoid(z)
    off = 4 * unit * (1 + X.abs())                        # of h, z and what is made of them, all of order 1 + |x|
    assert ((four(y) - z * sig).abs() <= off + store * (z * sig).abs()).all()
    d = four(dy) * sig * (1 + z * (1 - sig))
    u = d * W
    want = four(dy) + (u - u.mean((1, 3), keepdim=True) - h * (u * h).mean((1, 3), keepdim=True)) * r
    assert ((four(dx) - want).abs() <= (4 + four(dy).abs()) * off + store * want.abs()).all()
    for got, terms in ((dw, d * h), (db, d)):
        assert ((got.double().view(groups, -1) - terms.sum((0, 1))).abs() <= 8 * unit * (terms.abs() + four(dy).abs() * (1 + X.abs())).sum((0, 1))).all()
