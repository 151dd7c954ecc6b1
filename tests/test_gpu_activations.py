"""gelu, silu and their slopes, in bits: fp32 as good as elementary fp32 operations, and good in relation to themselves where they are small."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import operator_definitions as D  # noqa: E402
from paper_2505_14371_amd import operators as ops  # noqa: E402


@pytest.fixture(autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("a GPU test was selected but no GPU is visible")


def definition(z, activation, slope):
    """On tensors, in 64 bits."""
    z = z.double()
    phi, density, s = 0.5 * torch.special.erfc(-z / math.sqrt(2)), torch.exp(-z * z / 2) / math.sqrt(2 * math.pi), torch.sigmoid(z)
    return {("gelu", False): lambda: z * phi, ("gelu", True): lambda: phi + z * density,
            ("silu", False): lambda: z * s, ("silu", True): lambda: s * (1 + z * (1 - s))}[activation, slope]()


def elementary(z, activation, slope):
    """By torch's elementary operations in fp32."""
    if activation == "gelu":
        phi = 0.5 * (1 + torch.erf(z * (1 / math.sqrt(2))))
        return phi + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi)) if slope else z * phi
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s)) if slope else z * s


def kernels(z, activation, slope):
    if slope:
        return ops.dropout_grad(torch.ones_like(z), 0.0, 0, 0, pre=z, activation=activation)
    return ops.dropout(z, 0.0, 0, 0, activation=activation)


@pytest.mark.parametrize("slope", [False, True])
@pytest.mark.parametrize("activation", ["gelu", "silu"])
def test_fp32_is_as_good_as_elementary_operations(activation, slope):
    """Relative error in the square mean over normal values: at most a fifth above that of the elementary operations, which are each rounded once."""
    z = torch.randn(1 << 21, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    want = definition(z, activation, slope)
    off = lambda v: float((v.double() - want).square().mean().sqrt() / want.square().mean().sqrt())  # noqa: E731
    assert off(kernels(z, activation, slope)) <= 1.2 * off(elementary(z, activation, slope))


@pytest.mark.parametrize("activation", ["gelu", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_small_values_on_the_left_are_good_in_relation_to_themselves(activation, dtype):
    """z Phi(z) and z / (1 + exp(-z)) down to z = -12.  An error of half a unit of z, or of z^2, in the exponent's argument is one of z^2
    units of the value; a function of the library is good to a few units.  bf16: the store's half unit, and that far less."""
    z = -torch.logspace(-4, math.log10(12.0), 20001, device="cuda").to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype])
    want = definition(z, activation, False)
    relative = 2 * D.U32 * (z.double().square() + 8) if dtype == "f32" else D.STORE["bf16"] * 1.01
    got = kernels(z, activation, False).double()
    assert ((got - want).abs() <= relative * want.abs()).all(), float(((got - want) / want).abs().max())


@pytest.mark.parametrize("activation", ["gelu", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ends(activation, dtype):
    """Far out the functions are z and 0, their slopes 1 and 0; infinities and NaN go through the formulas."""
    far = torch.tensor([30.0, 200.0, 1e4, -200.0, -1e4], device="cuda").to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype])
    assert torch.equal(kernels(far, activation, False), far.clamp(min=0)) and torch.equal(kernels(far, activation, True), (far > 0).to(far.dtype))
    odd = torch.tensor([float("inf"), float("nan"), 0.0, -0.0], device="cuda").to(far.dtype)
    y, g = kernels(odd, activation, False), kernels(odd, activation, True)
    assert y[0] == float("inf") and y[1].isnan() and (y[2:] == 0).all()
    assert g[1].isnan() and (g[2:] == 0.5).all()
    assert np.isfinite(g[2:].double().cpu().numpy()).all()
