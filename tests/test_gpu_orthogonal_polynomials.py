"""Updates by polynomials other than the usual ones, against the formula in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

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
