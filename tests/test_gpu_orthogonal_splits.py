"""Updates whose symmetric products are taken by tiles of 96 with their sums in parts, which a join adds up: every entry that the join reads has to
have been written, so the workspace holds NaN.  Against the formula in 64 bits on the GPU."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import operator_definitions as D  # noqa: E402
from paper_2505_14371_amd import matrices as mats  # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
Q = mats.QUINTIC


@pytest.fixture(autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("a GPU test was selected but no GPU is visible")


def over_nan(g, steps):
    """orthogonalize(g) through the C interface, in a workspace of NaN."""
    n, rows, cols = g.shape
    x = torch.empty_like(g)
    args = mats._ORTHOGONALIZE.pack({torch.float32: 0, torch.bfloat16: 1}[g.dtype], steps, n, rows, cols, g.data_ptr(), rows * cols, cols, x.data_ptr(), rows * cols, cols, *Q, 1e-7)
    lib = mats._load()
    need = lib.qoda_orthogonalize_workspace_bytes(args)
    work = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    assert need > 0 and lib.qoda_orthogonalize(args, work.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == 0
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("steps", [1, 5])
@pytest.mark.parametrize("n,rows,cols", [(3, 672, 4000), (8, 480, 2048), (1, 1440, 2176), (1, 2176, 1440), (2, 541, 9000), (16, 290, 1500)])
def test_nothing_unwritten_is_read(n, rows, cols, steps, dtype):
    g = (torch.randn(n, rows, cols, device="cuda", generator=torch.Generator("cuda").manual_seed(rows + n)) * 1e-3).to(TYPES[dtype])
    got = over_nan(g, steps).double()
    assert torch.isfinite(got).all()
    x = g.double()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)
    for _ in range(steps):
        s = torch.matmul(x, x.transpose(1, 2).contiguous()) if rows <= cols else torch.matmul(x.transpose(1, 2).contiguous(), x)
        p = Q[1] * s + Q[2] * torch.matmul(s, s)
        x = Q[0] * x + (torch.matmul(p, x) if rows <= cols else torch.matmul(x, p))
    # A step is off by 2^-22 (a pair) and 2^-24 root(k) (a sum) of X's norm for each of the operands and terms of its three products, fewer than 16; X's norm is 1 at first, and it and
    # what is off grow by less than 3.4445 a step.
    norm = x.flatten(1).norm(dim=1)
    off = (got - x).flatten(1).norm(dim=1)
    bound = 16 * steps * 3.4445 ** (steps - 1) * (2.0**-22 + max(rows, cols) ** 0.5 * 2.0**-24)
    assert (off <= bound + D.STORE[dtype] * 1.01 * norm).all(), (off / norm)
    assert torch.equal(over_nan(g, steps).double(), got)
