"""Group normalisation of samples without positions or channels: its statistics are those of no values, not what the memory held."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2505_14371_amd import operators as ops  # noqa: E402


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("shape,groups", [((3, 0, 8), 2), ((2, 4, 0), 1), ((5, 0), 3), ((2, 3, 0, 16), 4)])
def test_statistics_of_no_values_are_nan(shape, groups, native, monkeypatch):
    if not torch.cuda.is_available():
        pytest.fail("a GPU test was selected but no GPU is visible")
    if not native:
        monkeypatch.setattr(ops, "_native", None)
    x = torch.empty(shape, device="cuda")
    held = [torch.full((shape[0], groups), 7.0, device="cuda") for _ in range(8)]     # what their memory holds next
    del held
    y, mean, rstd = ops.group_norm(x, groups)
    assert y.shape == x.shape and mean.shape == rstd.shape == (shape[0], groups)
    assert mean.isnan().all() and rstd.isnan().all()
