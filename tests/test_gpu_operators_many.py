"""Operators of more rows, groups and columns than one launch takes (fewer than 2^32 work-items): every part of the outputs is that of its own rows."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2505_14371_amd import operators as ops  # noqa: E402


@pytest.fixture(autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("a GPU test was selected but no GPU is visible")
    yield
    torch.cuda.empty_cache()


def random(*shape):
    return torch.randn(shape, device="cuda", dtype=torch.bfloat16, generator=torch.Generator(device="cuda").manual_seed(1))


def around(n, most):
    """The first of n, those on both sides of where a launch ends, and the last."""
    return [(0, 40), (most - 40, min(most + 40, n)), (n - 40, n)]


@pytest.mark.parametrize("n,s,c,a_workgroup", [((1 << 28) + 5, 1, 8, 16), ((1 << 26) + 3, 2, 1, None)])
def test_samples_of_a_norm(n, s, c, a_workgroup):
    """Rows in teams of 16 lanes; maps in workgroups of 64."""
    most = ((1 << 32) - 1) // 256 * a_workgroup if a_workgroup else ((1 << 32) - 1) // 64
    x = random(n, s, c)
    y, mean, rstd = ops.group_norm(x, 1, eps=1e-3)
    dx, dw, db = ops.group_norm_grad(y, x, mean, rstd, 1, residual=x)
    for a, b in around(n, most):
        y1, mean1, rstd1 = ops.group_norm(x[a:b], 1, eps=1e-3)
        assert torch.equal(y[a:b], y1) and torch.equal(mean[a:b], mean1) and torch.equal(rstd[a:b], rstd1)
        assert torch.equal(dx[a:b], ops.group_norm_grad(y1, x[a:b], mean1, rstd1, 1, residual=x[a:b])[0])
    # the sums of n s terms of order 1, joined from a few thousand partial sums
    want = torch.stack([y[i: i + (1 << 24)].double().sum((0, 1)) for i in range(0, n, 1 << 24)]).sum(0)
    assert ((db.double() - want).abs() <= 1e-5 * n * s).all()


def test_groups_of_a_norm():
    groups, len = (1 << 24) + 5, 2
    x, dy = random(1, groups * len), random(1, groups * len).flip(1)
    y, mean, rstd = ops.group_norm(x, groups, activation="silu")
    dx, dw, db = ops.group_norm_grad(dy, x, mean, rstd, groups, activation="silu")
    # launches of a workgroup a group, and of one for 16 of the columns of sums, dweight's and then dbias's
    columns = ((1 << 32) - 1) // 1024 * 16 - groups * len
    assert 0 < columns < groups * len
    for a, b in around(groups, ((1 << 32) - 1) // 256) + around(groups, columns // len):
        part = slice(a * len, b * len)
        y1, mean1, rstd1 = ops.group_norm(x[:, part], b - a, activation="silu")
        assert torch.equal(y[:, part], y1) and torch.equal(mean[:, a:b], mean1)
        dx1, dw1, db1 = ops.group_norm_grad(dy[:, part], x[:, part], mean1, rstd1, b - a, activation="silu")
        assert torch.equal(dx[:, part], dx1) and torch.equal(dw[part], dw1) and torch.equal(db[part], db1)
    # with one sample and without weights the sums are the terms themselves
    z = (x.float() - mean.repeat_interleave(len, 1)) * rstd.repeat_interleave(len, 1)
    sig = torch.sigmoid(z)
    want = dy.float() * sig * (1 + z * (1 - sig))
    assert ((db - want[0]).abs() <= 1e-5 * (1 + want[0].abs())).all() and ((dw - (want * z)[0]).abs() <= 1e-5 * (1 + want[0].abs())).all()


def test_one_row_by_many():
    n = (1 << 28) + 40
    w, x = random(n, 1), torch.full((1, 1), -1.5, device="cuda", dtype=torch.bfloat16)
    assert torch.equal(ops.linear(x, w)[0], w[:, 0] * -1.5)           # a product of two bf16 is exact before it is stored


def test_many_rows_by_one():
    n = (1 << 30) + 100
    x, w = random(n, 1), torch.full((1, 1), 0.75, device="cuda", dtype=torch.bfloat16)
    assert torch.equal(ops.linear(x, w), x * 0.75)
