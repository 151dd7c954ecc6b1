"""Tensors that torch is to differentiate, and tangents, in the calls on matrices in four bits and on updates: none is lost in silence where a derivative could be asked for."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2505_14371_amd import matrices as mats  # noqa: E402
from paper_2505_14371_amd import operators as ops  # noqa: E402

ad = torch.autograd.forward_ad


@pytest.fixture(autouse=True, params=["native", "python"])
def look(request, monkeypatch):
    if not torch.cuda.is_available():
        pytest.fail("a GPU test was selected but no GPU is visible")
    mats._load()
    if request.param == "python":
        monkeypatch.setattr(ops, "_native", None)
        monkeypatch.setattr(mats, "_native", None)


def weight(cout=4, cin=8):
    return mats.microscale(torch.ones((cout, cin), device="cuda"))


LINEAR = {"x": lambda t: mats.mx_linear(t, weight(), keep_pre=True)[1], "one row": lambda t: mats.mx_linear(t[0], weight()),
          "residual": lambda t: mats.mx_linear(torch.ones((3, 8), device="cuda"), weight(8), residual=t),
          "bias": lambda t: mats.mx_linear(torch.ones((3, 8), device="cuda"), weight(24), t.flatten()),
          "microscaled x, residual": lambda t: mats.mx_linear(weight(3), weight(8), residual=t, dtype=torch.float32)}
REFUSED = {"microscale": lambda t: mats.microscale(t), "microscale: transposed": lambda t: mats.microscale(t, transposed=True, rounding="stochastic"),
           "orthogonalize": lambda t: mats.orthogonalize(t), "orthogonalize: out": lambda t: mats.orthogonalize(torch.ones((3, 8), device="cuda"), out=t)}


@pytest.mark.parametrize("name", LINEAR)
def test_a_derivative_that_is_not_recorded_is_not_lost_in_silence(name):
    x = torch.randn((3, 8), device="cuda")
    want = LINEAR[name](x)
    assert not want.requires_grad
    x.requires_grad_()
    y = LINEAR[name](x)
    assert torch.equal(y, want) and y.requires_grad
    with pytest.raises(RuntimeError, match="mx_linear records nothing"):
        (y.sum() + x.sum()).backward()
    with torch.no_grad():
        assert not LINEAR[name](x).requires_grad
    assert not LINEAR[name](x.detach()).requires_grad


@pytest.mark.parametrize("name", REFUSED)
def test_what_has_no_gradient_call_refuses_at_once(name):
    x = torch.randn((3, 8), device="cuda", requires_grad=True)
    with pytest.raises(RuntimeError, match=name.split(":")[0]):
        REFUSED[name](x)
    with torch.no_grad():
        REFUSED[name](x)
    REFUSED[name](x.detach())


@pytest.mark.parametrize("name", [*LINEAR, *REFUSED])
def test_a_tangent_is_refused(name):
    x = torch.randn((3, 8), device="cuda")
    call = {**LINEAR, **REFUSED}[name]
    with ad.dual_level():
        dual = ad.make_dual(x, torch.ones_like(x))
        with pytest.raises(RuntimeError):
            call(dual)
        with torch.no_grad(), pytest.raises(RuntimeError):
            call(dual)
        call(x)


def test_gradient_calls_return_plain_tensors():
    x = torch.randn((3, 8), device="cuda", requires_grad=True)
    w = mats.microscale(torch.ones((8, 8), device="cuda"))
    for got in (mats.mx_linear_input_grad(x, w), mats.mx_linear_input_grad(x, w, pre=x, activation="gelu", residual=x)):
        assert not got.requires_grad
    want = mats.mx_linear_input_grad(x.detach(), w, pre=x.detach(), activation="gelu", residual=x.detach())
    assert torch.equal(mats.mx_linear_input_grad(x, w, pre=x, activation="gelu", residual=x), want)
    dw, db = mats.mx_linear_weight_grad(weight(), weight(5))
    assert not dw.requires_grad and not db.requires_grad


def test_under_autograd_as_a_function_of_its_own():
    """The calls where they belong: in a Function's forward and backward."""
    class Linear(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w):
            ctx.save_for_backward(x, w)
            return mats.mx_linear(x, mats.microscale(w))

        @staticmethod
        def backward(ctx, dy):
            x, w = ctx.saved_tensors
            return (mats.mx_linear_input_grad(dy, mats.microscale(w, transposed=True)),
                    mats.mx_linear_weight_grad(mats.microscale(dy, transposed=True), mats.microscale(x, transposed=True), bias=False)[0])

    x, w = torch.randn((3, 8), device="cuda", requires_grad=True), torch.randn((4, 8), device="cuda", requires_grad=True)
    y = Linear.apply(x, w)
    dy = torch.randn_like(y)
    y.backward(dy)
    assert torch.equal(x.grad, mats.mx_linear_input_grad(dy, mats.microscale(w.detach(), transposed=True)))
    assert torch.equal(w.grad, mats.mx_linear_weight_grad(mats.microscale(dy, transposed=True), mats.microscale(x.detach(), transposed=True))[0])
