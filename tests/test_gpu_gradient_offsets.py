"""Gradients of matrices and maps of more than 2^31 entries and 4 GB: what lies behind is right, and what has no gradient in front adds nothing."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2505_14371_amd import operators as ops  # noqa: E402

ROWS, COLS, TAIL = 65600, 32776, 64


@pytest.fixture(autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("a GPU test was selected but no GPU is visible")
    yield
    torch.cuda.empty_cache()


def tailed(*shape, last=TAIL):
    """Zeros, behind them normal values."""
    t = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
    t[-last:] = torch.randn((last, *shape[1:]), device="cuda", generator=torch.Generator(device="cuda").manual_seed(shape[-1])).to(torch.bfloat16)
    return t


def test_of_dropout():
    dy, pre = tailed(ROWS, COLS), tailed(ROWS, COLS)
    dz = ops.dropout_grad(dy, 0.0, 1, 2, pre=pre, activation="gelu")
    assert torch.equal(dz[-TAIL:], ops.dropout_grad(dy[-TAIL:], 0.0, 1, 2, pre=pre[-TAIL:], activation="gelu"))
    assert not dz[:TAIL].any() and dz[-TAIL:].any()


def test_of_products():
    w, dz = (torch.randn((24, COLS), device="cuda") / 5).to(torch.bfloat16), tailed(ROWS, 24)
    pre = tailed(ROWS, COLS)
    dx = ops.linear_input_grad(dz, w, pre=pre, activation="silu", residual=pre)
    part = ops.linear_input_grad(dz[-TAIL:], w, pre=pre[-TAIL:], activation="silu", residual=pre[-TAIL:])
    assert torch.allclose(dx[-TAIL:].float(), part.float(), rtol=2**-7, atol=1e-5) and not dx[:TAIL].any()     # sums of 24 terms, cut alike or not
    del dx
    dw, db = ops.linear_weight_grad(dz, pre)
    dw1, db1 = ops.linear_weight_grad(dz[-TAIL:], pre[-TAIL:])
    assert torch.allclose(dw, dw1, rtol=1e-5, atol=1e-4) and torch.allclose(db, db1, rtol=1e-5, atol=1e-4)     # 64 terms of order 1


def test_of_a_norm_of_rows():
    x, dy = tailed(ROWS, COLS), tailed(ROWS, COLS)
    y, mean, rstd = ops.group_norm(x, 4, activation="gelu")
    dx, dw, db = ops.group_norm_grad(dy, x, mean, rstd, 4, activation="gelu")
    last = [t[-TAIL:] for t in (dy, x, mean, rstd)]
    dx1, dw1, db1 = ops.group_norm_grad(*last, 4, activation="gelu")
    assert torch.equal(dx[-TAIL:], dx1) and not dx[:TAIL].any()
    assert torch.allclose(dw, dw1, rtol=1e-5, atol=1e-4) and torch.allclose(db, db1, rtol=1e-5, atol=1e-4)


@pytest.mark.parametrize("groups", [32, 64])     # groups wider than a block, and narrower of an odd width
def test_of_a_norm_of_maps(groups):
    x, dy = tailed(4, 8200, 65600, last=1), tailed(4, 8200, 65600, last=1)
    y, mean, rstd = ops.group_norm(x, groups)
    y1, mean1, rstd1 = ops.group_norm(x[-1:], groups)
    assert torch.equal(y[-1:], y1) and torch.equal(mean[-1:], mean1) and torch.equal(rstd[-1:], rstd1) and not y[0].any()
    del y, y1
    dx, dw, db = ops.group_norm_grad(dy, x, mean, rstd, groups)
    dx1, dw1, db1 = ops.group_norm_grad(dy[-1:], x[-1:], mean1, rstd1, groups)
    assert torch.equal(dx[-1:], dx1) and not dx[0].any()
    assert torch.allclose(dw, dw1, rtol=1e-5, atol=1e-2) and torch.allclose(db, db1, rtol=1e-5, atol=1e-2)     # 8200 terms of order 1
