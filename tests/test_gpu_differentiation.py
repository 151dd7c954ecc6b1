"""Tensors that torch is to differentiate: the operators record no derivative, and say so where one is asked for."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2505_14371_amd import operators as ops  # noqa: E402

FORWARD = {"linear": lambda x: ops.linear(x, torch.ones((4, 8), device="cuda"), keep_pre=True)[0],
           "linear: residual": lambda x: ops.linear(torch.ones((3, 8), device="cuda"), torch.ones((8, 8), device="cuda"), residual=x),
           "dropout": lambda x: ops.dropout(x, 0.0, 1, 1), "group_norm": lambda x: ops.group_norm(x, 2)[0]}


@pytest.fixture(autouse=True, params=["native", "python"])
def look(request, monkeypatch):
    if not torch.cuda.is_available():
        pytest.fail("a GPU test was selected but no GPU is visible")
    if request.param == "python":
        monkeypatch.setattr(ops, "_native", None)


@pytest.mark.parametrize("name", FORWARD)
def test_a_derivative_that_is_not_recorded_is_not_lost_in_silence(name):
    x = torch.randn((3, 8), device="cuda")
    want = FORWARD[name](x)
    assert not want.requires_grad
    x.requires_grad_()
    y = FORWARD[name](x)
    assert torch.equal(y, want) and y.requires_grad
    with pytest.raises(RuntimeError, match=name.split(":")[0]):
        (y.sum() + x.sum()).backward()                # x.sum() alone would have given x a gradient
    with torch.no_grad():
        assert not FORWARD[name](x).requires_grad
    assert not FORWARD[name](x.detach()).requires_grad
    w = torch.nn.Parameter(torch.ones((4, 8), device="cuda"))
    assert ops.linear(x.detach(), w).requires_grad


@pytest.mark.parametrize("name", FORWARD)
def test_a_tangent_is_refused(name):
    x = torch.randn((3, 8), device="cuda")
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(x, torch.ones_like(x))
        with pytest.raises(RuntimeError, match=name.split(":")[0]):
            FORWARD[name](dual)


def test_gradient_calls_return_plain_tensors():
    x, w = torch.nn.Parameter(torch.randn((3, 8), device="cuda")), torch.nn.Parameter(torch.randn((8, 8), device="cuda"))
    assert not ops.linear_input_grad(x, w).requires_grad and not ops.linear_weight_grad(x, x)[0].requires_grad
    assert not ops.dropout_grad(x, 0.5, 1, 1).requires_grad
