"""Updates whose result lies in g's memory: g itself and what is apart from it are taken, anything between is refused."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2505_14371_amd import matrices as mats  # noqa: E402
from paper_2505_14371_amd import qoda  # noqa: E402


@pytest.mark.parametrize("rows,cols", [(40, 50), (50, 40), (300, 410)])
def test_views_of_one_buffer(rows, cols):
    buf = torch.randn(6, rows, 2 * cols, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    g = buf[:3, :, :cols]
    was, want = buf.clone(), mats.orthogonalize(g.contiguous())
    for out in (buf[1:4, :, :cols], buf[:3, :, 1: cols + 1], buf[2:5, :, cols - 1: 2 * cols - 1], buf.flatten()[7: 7 + 3 * rows * cols].view(3, rows, cols)):
        with pytest.raises(qoda.QodaError, match="neither g nor apart"):
            mats.orthogonalize(g, out=out)
    assert torch.equal(buf, was)
    for out in (buf[:3, :, cols:], buf[3:, :, :cols], buf[3:, :, cols:]):
        assert mats.orthogonalize(g, out=out) is out and torch.equal(out, want) and torch.equal(g, was[:3, :, :cols])
    assert torch.equal(mats.orthogonalize(g, out=g), want)
    again = was[0]
    want = mats.orthogonalize(again)
    assert torch.equal(mats.orthogonalize(again, out=again.view(again.shape)), want) and torch.equal(again, want)
