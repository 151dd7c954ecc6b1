"""The gradient of a normalisation through relu and leaky_relu: on the side of the kink that the forward pass took, and by the formula."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import operator_definitions as D  # noqa: E402
from paper_2505_14371_amd import operators as ops  # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# rows of one, four and many eights a lane; maps of a wave, of a workgroup, in pieces, of groups wider than a block; odd widths
SHAPES = [(3000, 1, 96, 1), (500, 1, 2048, 1), (9, 1, 8200, 2), (700, 9, 24, 3), (40, 256, 64, 8), (3, 1000, 130, 13), (2, 5000, 64, 2), (2, 3000, 26, 2), (1, 300, 4100, 1)]


@pytest.fixture(autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("a GPU test was selected but no GPU is visible")


def inputs(n, s, c, far, dtype):
    gen = torch.Generator(device="cuda").manual_seed(n + s + c)
    draw = lambda *shape: torch.randn(shape, device="cuda", generator=gen)  # noqa: E731
    return (far + draw(n, s, c)).to(TYPES[dtype]), 1 + 0.2 * draw(c), 0.2 * draw(c), draw(n, s, c).to(TYPES[dtype])


@pytest.mark.parametrize("dtype,far", [("f32", 0.0), ("f32", 4096.0), ("bf16", 16.0)])
@pytest.mark.parametrize("activation", ["relu", "leaky_relu"])
@pytest.mark.parametrize("n,s,c,groups", SHAPES)
def test_gradient_takes_the_side_that_the_forward_took(n, s, c, groups, activation, dtype, far):
    """With dy = 5 a channel's dbias is 5 for each of its positive outputs and 0 or (5 times 0.2, in fp32) 1 for each other: whole
    numbers below 2^24, so exact in any order."""
    x, w, b, _ = inputs(n, s, c, far, dtype)
    y, mean, rstd = ops.group_norm(x, groups, w, b, activation=activation)
    _, _, db = ops.group_norm_grad(torch.full_like(x, 5.0), x, mean, rstd, groups, w, b, activation=activation)
    positive = (y > 0).sum((0, 1))
    assert torch.equal(db.double(), (5 * positive + (n * s - positive if activation == "leaky_relu" else 0)).double())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("activation", ["relu", "leaky_relu"])
@pytest.mark.parametrize("n,s,c,groups", SHAPES)
def test_gradient_through_a_kink(n, s, c, groups, activation, dtype, monkeypatch):
    """Against the formula in 64 bits, the slope at each entry that of the forward pass's own side."""
    x, w, b, dy = inputs(n, s, c, 1.0, dtype)
    y, mean, rstd = ops.group_norm(x, groups, w, b, activation=activation)
    got = ops.group_norm_grad(dy, x, mean, rstd, groups, w, b, activation=activation)
    wide = [t.double().cpu().numpy() for t in (dy, x, mean, rstd, w, b)]
    side = np.where((y > 0).cpu().numpy(), 1.0, 0.2 if activation == "leaky_relu" else 0.0)
    monkeypatch.setattr(D, "slope", lambda z, a: side)
    want = D.group_norm_grad(*wide[:4], groups, *wide[4:], activation)
    # sums of k terms of fp32, in trees of at most a few hundred one after the other; entries of dx are of order 1, their terms below 60
    k = max(n * s, s * c // groups)
    for g, e, store in zip(got, want, (D.STORE[dtype], 0.0, 0.0)):
        g = g.double().cpu().numpy()
        scale = np.abs(wide[0]).max() * (1 + np.abs(wide[1]).max()) * 4
        bound = 2 * D.U32 * scale * (16 + min(k, 2000)) + np.abs(e) * (store * 1.001 + 2 * D.U32 * 16) if store else 2 * D.U32 * scale * (16 + np.sqrt(k) * 16)
        assert (np.abs(g - e) <= bound).all(), (np.abs(g - e).max(), np.max(bound))
