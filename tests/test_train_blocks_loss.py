"""The loss that the blocks' training run prints and the gradient that it trains by belong together (CPU)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2505_14371_amd.harness import train_blocks  # noqa: E402


@pytest.mark.parametrize("shape", [(7, 5), (1, 1), (2, 3, 4)])
def test_gradient_is_that_of_the_loss(shape):
    gen = torch.Generator().manual_seed(1)
    y, target = (torch.randn(shape, generator=gen, dtype=torch.float32) for _ in range(2))
    y.requires_grad_()
    loss, dy = train_blocks.loss_of(y, target)
    loss.backward()
    assert torch.allclose(dy, y.grad, rtol=1e-6, atol=1e-7)      # two roundings of fp32
    assert train_blocks.loss_of(y.detach().to(torch.bfloat16), target)[1].dtype == torch.bfloat16
