"""The operators of include/qoda_matrices.h as they are used: residual blocks in four bits, orthogonalised dual vectors, captured graphs, other streams,
several threads, and matrices of more than 2^31 entries."""
import threading

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import matrix_definitions as M  # noqa: E402
import operator_definitions as D  # noqa: E402
from paper_2505_14371_amd import matrices as mats  # noqa: E402
from paper_2505_14371_amd import operators as ops  # noqa: E402
from paper_2505_14371_amd.blocks import ResidualBlocks  # noqa: E402
from paper_2505_14371_amd.harness import train_blocks  # noqa: E402


@pytest.fixture(autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("a GPU test was selected but no GPU is visible")


wide = lambda t: t.double().cpu().numpy()  # noqa: E731


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,p", [(70, 0.1), (5, 0.0)])
def test_a_block_in_four_bits(rows, p, dtype):
    """One block, forward and backward, each product against its formula from the operands that it had."""
    model = ResidualBlocks(60, 200, 1, p=p, dtype={"bf16": torch.bfloat16, "f32": torch.float32}[dtype], seed=3, four_bit=True)
    gamma, beta, w1, b1, w2, b2 = model.params
    gen = torch.Generator("cuda").manual_seed(1)
    x, dy = (torch.randn((rows, 60), device="cuda", generator=gen).to(model.dtype) for _ in range(2))
    weights, grads = model.weights(), model.gradients()
    y, saved = model.forward(x, weights, draw=5)
    dx = model.backward(dy, saved, weights, grads)
    h, n, mean, rstd, z, a = saved[1]
    drop = [(10, p), (11, p)]                     # offsets of the two sites: draw depth 2 + site
    r1, r2, t1, t2 = M.rounded(wide(w1)), M.rounded(wide(w2)), M.rounded(wide(w1).T).T, M.rounded(wide(w2).T).T
    near = lambda got, want, bound: np.testing.assert_array_less(np.abs(wide(got) - want), D.stored(bound, want, dtype) + 1e-30)  # noqa: E731
    scale = 1 / (1 - p) * 1.01
    bz = D.sum_bound(60, np.abs(M.rounded(wide(n))) @ np.abs(r1).T + np.abs(wide(b1)))
    zw = M.rounded(wide(n)) @ r1.T + wide(b1)
    near(z, zw, bz)
    near(a, D.drop(D.act(zw, "gelu"), p, 3, drop[0][0]), scale * (1.13 * bz + D.ACT_ERROR * (1 + np.abs(zw))))
    ya = M.rounded(wide(a))
    near(y, wide(x) + D.drop(ya @ r2.T + wide(b2), p, 3, drop[1][0]), scale * D.sum_bound(200, np.abs(ya) @ np.abs(r2).T + np.abs(wide(b2))) + 4 * D.U32 * (np.abs(wide(x)) + 9))
    d2 = wide(ops.dropout_grad(dy, p, 3, drop[1][0]))
    q, qt = M.rounded(d2, True, 3, 2 * drop[1][0]), M.rounded(d2.T, True, 3, 2 * drop[1][0] + 1)
    at = M.rounded(wide(a).T)
    exact = lambda got, want, bound: np.testing.assert_array_less(np.abs(wide(got) - want), bound + 1e-30)  # noqa: E731
    exact(grads[4], qt @ at.T, D.sum_bound(rows, np.abs(qt) @ np.abs(at).T) + 1e-7 * np.abs(qt @ at.T))
    exact(grads[5], qt.sum(1), D.sum_bound(rows, np.abs(qt).sum(1)) + 1e-7 * np.abs(qt.sum(1)))
    zb = wide(z)
    d1 = D.drop(q @ t2 * D.slope(zb, "gelu"), p, 3, drop[0][0])
    got = mats.mx_linear_input_grad(mats.microscale(ops.dropout_grad(dy, p, 3, drop[1][0]), rounding="stochastic", seed=3, offset=2 * drop[1][0]), weights[1][1], pre=z,
                                    activation="gelu", p=p, seed=3, offset=drop[0][0], dtype=model.dtype)
    near(got, d1, scale * (1.13 * D.sum_bound(60, np.abs(q) @ np.abs(t2)) + D.ACT_ERROR * (1 + np.abs(zb)) * np.abs(q @ t2)))
    g = wide(got)
    gt, nt = M.rounded(g.T, True, 3, 2 * drop[0][0] + 1), M.rounded(wide(n).T)
    exact(grads[2], gt @ nt.T, D.sum_bound(rows, np.abs(gt) @ np.abs(nt).T) + 1e-7 * np.abs(gt @ nt.T))
    exact(grads[3], gt.sum(1), D.sum_bound(rows, np.abs(gt).sum(1)) + 1e-7 * np.abs(gt.sum(1)))
    dn = mats.mx_linear_input_grad(mats.microscale(got, rounding="stochastic", seed=3, offset=2 * drop[0][0]), weights[0][1], dtype=model.dtype)
    want = ops.group_norm_grad(dn, h, mean, rstd, 1, gamma, beta, residual=dy)[0]
    assert torch.equal(dx, want)
    once = [v.clone() for v in grads]
    model.backward(dy, saved, weights, grads, accumulate=True)
    for v, o in zip(grads, once):
        assert torch.allclose(v, 2 * o, rtol=1e-5, atol=1e-5 * float(o.abs().max()))


def test_the_mean_gradient_in_four_bits_is_that_of_the_rounded_operands():
    """Stochastic rounding: over many draws the weight gradient's mean nears the product with the unrounded dz, to six deviations of the mean."""
    gen = torch.Generator("cuda").manual_seed(1)
    dz, x = torch.randn((96, 40), device="cuda", generator=gen), mats.microscale(torch.randn((96, 50), device="cuda", generator=gen), transposed=True)
    runs = torch.stack([mats.mx_linear_weight_grad(mats.microscale(dz, transposed=True, rounding="stochastic", seed=2, offset=k), x, bias=False)[0] for k in range(400)]).double()
    want = torch.matmul(dz.t().double().contiguous(), x.values().double().t().contiguous())
    off = (runs.mean(0) - want).abs() / (runs.std(0) / 20 + 1e-4)
    assert off.max() < 6, off.max()


@pytest.mark.parametrize("depth", [1, 3])
def test_gradients_of_matrices_are_orthogonalised_in_place(depth):
    model = ResidualBlocks(48, 96, depth, p=0.0, seed=1)
    flat, apart = model.gradients(), None
    for g in flat:
        g.copy_(torch.randn(g.shape, device="cuda"))
    apart = [g.clone() for g in flat]
    want = [mats.orthogonalize(g, steps=4) if g.dim() == 2 else g.clone() for g in flat]
    model.orthogonalize(flat, steps=4)
    model.orthogonalize(apart, steps=4)          # tensors of their own, not evenly spaced
    for a, b, w in zip(flat, apart, want):
        assert torch.equal(a, w) and torch.equal(b, w)


@pytest.mark.parametrize("four_bit,orthogonal", [(True, False), (False, True), (True, True)])
def test_training_runs(four_bit, orthogonal):
    losses, _, _ = train_blocks.train(width=64, hidden=128, depth=2, nodes=3, rows=256, rounds=5, four_bit=four_bit, orthogonal=orthogonal)
    assert len(losses) == 5 and all(np.isfinite(losses))


def everything(x, dz, w, g, out):
    """A training step's calls on these operands, their results written into `out`."""
    wq, wt = mats.microscale(w), mats.microscale(w, transposed=True)
    y, z = mats.mx_linear(x, wq, activation="gelu", p=0.1, seed=1, offset=2, keep_pre=True)
    dx = mats.mx_linear_input_grad(mats.microscale(dz, rounding="stochastic", seed=1, offset=3), wt, dtype=x.dtype)
    dw, db = mats.mx_linear_weight_grad(mats.microscale(dz, transposed=True, rounding="stochastic", seed=1, offset=4), mats.microscale(x, transposed=True))
    one = mats.mx_linear(x[0], wq)
    for o, r in zip(out, (y, z, dx, dw, db, one, mats.orthogonalize(dw), mats.orthogonalize(g), wq.values())):
        o.copy_(r)


def operands(rows, cin, cout, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    draw = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    x, dz, w, g = draw(rows, cin).bfloat16(), draw(rows, cout).bfloat16(), draw(cout, cin), draw(3, 40, 50)
    out = [torch.zeros(s, dtype=t, device="cuda") for s, t in (((rows, cout), torch.bfloat16), ((rows, cout), torch.bfloat16), ((rows, cin), torch.bfloat16), ((cout, cin), torch.float32),
                                                             ((cout,), torch.float32), ((cout,), torch.bfloat16), ((cout, cin), torch.float32), ((3, 40, 50), torch.float32), ((cout, cin), torch.float32))]
    return x, dz, w, g, out


@pytest.mark.parametrize("rows,cin,cout", [(40, 300, 200), (3000, 130, 300)])
def test_captured_and_replayed(rows, cin, cout):
    """A graph of the calls, replayed on new operands with eager work in between, gives what the calls give."""
    x, dz, w, g, out = operands(rows, cin, cout, 1)
    everything(x, dz, w, g, out)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        everything(x, dz, w, g, out)
    for k in range(4):
        x2, dz2, w2, g2, want = operands(rows, cin, cout, 10 + k)
        everything(x2, dz2, w2, g2, want)
        for a, b in zip((x, dz, w, g), (x2, dz2, w2, g2)):
            a.copy_(b)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), k


def test_two_graphs_of_the_same_operands_replayed_in_turn():
    """Each has workspaces of its own."""
    a, b = operands(600, 500, 300, 1), operands(600, 500, 300, 2)
    want = [[torch.zeros_like(o) for o in v[4]] for v in (a, b)]
    for v, o in zip((a, b), want):
        everything(*v[:4], o)
    graphs = []
    for v in (a, b):
        everything(*v)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            everything(*v)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(3):
        for v in (a, b):
            for o in v[4]:
                o.zero_()
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for v, o in zip((a, b), want):
            assert all(torch.equal(p, q) for p, q in zip(v[4], o))


def test_on_a_stream_that_is_named():
    x, w, g = torch.randn(500, 300, device="cuda"), torch.randn(200, 300, device="cuda"), torch.randn(300, 200, device="cuda")
    wq = mats.microscale(w)
    want = (mats.mx_linear(x, wq), mats.microscale(x, transposed=True).values(), mats.orthogonalize(g), mats.mx_linear_input_grad(x, wq), mats.mx_linear_weight_grad(wq, mats.microscale(x))[0])
    torch.cuda.synchronize()
    for s in (torch.cuda.Stream(), torch.cuda.Stream().cuda_stream):
        got = (mats.mx_linear(x, wq, stream=s), mats.microscale(x, transposed=True, stream=s).values(stream=s), mats.orthogonalize(g, stream=s), mats.mx_linear_input_grad(x, wq, stream=s),
               mats.mx_linear_weight_grad(wq, mats.microscale(x, stream=s), stream=s)[0])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_calls_from_several_threads():
    v = operands(300, 200, 100, 1)
    want = [torch.zeros_like(o) for o in v[4]]
    everything(*v[:4], want)
    torch.cuda.synchronize()
    outs, failed = [[torch.zeros_like(o) for o in want] for _ in range(4)], []

    def run(out):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    everything(*v[:4], out)
                with pytest.raises(ValueError):
                    mats.mx_linear(v[0][:, :7], mats.microscale(v[2]))
            torch.cuda.current_stream().synchronize()
        except BaseException as e:  # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=run, args=(o,)) for o in outs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    assert all(torch.equal(a, b) for out in outs for a, b in zip(out, want))


def test_more_than_2_31_entries():
    """Offsets of 64 bits: the last rows of matrices of 2.3 G entries against those rows by themselves."""
    rows, cols = 70016, 32800
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    for r in range(0, rows, 8752):
        x[r: r + 8752] = torch.randn((min(8752, rows - r), cols), device="cuda")
    tail = x[rows - 128:]
    q = mats.microscale(x)
    few = mats.microscale(tail)
    assert torch.equal(q.codes[rows - 128:], few.codes) and torch.equal(q.scales[:, -2:], few.scales)
    assert torch.equal(mats.Microscaled(q.codes[rows - 128:], q.scales[:, -2:].contiguous(), 128, cols).values(), few.values())
    values = q.values(torch.bfloat16)
    assert torch.equal(values[rows - 128:], few.values(torch.bfloat16))
    del values
    t = mats.microscale(x, transposed=True)          # columns of x, blocks along its 70016 rows: 273 steps and a half
    assert torch.equal(t.codes[cols - 32:, -128:-64], mats.microscale(x[rows - 128:, cols - 32:], transposed=True).codes[:, :64])
    del t
    w = mats.microscale(torch.randn(33000, 64, device="cuda"))
    a = torch.randn(70000, 64, device="cuda").bfloat16()
    y = mats.mx_linear(a, w)                         # 2.3 G sums
    assert torch.equal(y[-100:], mats.mx_linear(a[-100:], w)) and torch.equal(y[:100], mats.mx_linear(a[:100], w))


def test_more_than_2_30_rows():
    """Scales lie 256 bytes for 64 rows: those of the last rows are more than 2^32 bytes behind the first."""
    rows = 2**30 + 200
    x = torch.empty((rows, 1), dtype=torch.bfloat16, device="cuda").normal_()
    w = mats.microscale(torch.tensor([[1.0], [2.0], [-0.5]], device="cuda"))
    q = mats.microscale(x)
    y = mats.mx_linear(q, w)
    assert torch.equal(y[-300:], mats.mx_linear(x[-300:], w)) and torch.equal(y[:300], mats.mx_linear(x[:300], w))
    few = mats.mx_linear(w, q, dtype=torch.bfloat16)           # the many rows as the second operand, three of the first
    assert torch.equal(few[:, -300:], y[-300:].t()) and torch.equal(few[:, :300], y[:300].t())
    del few, y
    wide = mats.mx_linear(mats.microscale(torch.randn(20, 1, device="cuda")), q, dtype=torch.bfloat16)
    assert torch.isfinite(wide[:, -300:]).all()
    assert torch.equal(q.values(torch.bfloat16)[-300:], mats.microscale(x[-300:]).values(torch.bfloat16))


@pytest.mark.parametrize("rows,dtype,turned", [(130, torch.float32, False), (130, torch.float32, True), (2048, torch.bfloat16, False)])
def test_the_longest_side(rows, dtype, turned):
    """2^22 columns of which 300 are not zero, the last ones among them: the update is that of these 300."""
    cols = 2**22
    gen = torch.Generator("cuda").manual_seed(rows)
    few = torch.randn((rows, 300), device="cuda", generator=gen).to(dtype)
    at = list(range(7, cols - 20000, 20971)) + list(range(cols - 100, cols))
    g = torch.zeros((cols, rows) if turned else (rows, cols), dtype=dtype, device="cuda")
    columns = g.t() if turned else g
    assert len(at) == 300
    for i, j in enumerate(at):
        columns[:, j] = few[:, i]
    mats.orthogonalize(g, steps=1, out=g)
    got = torch.stack([columns[:, j] for j in at], 1)
    want = mats.orthogonalize(few, steps=1)
    # A's sums in another order, 2^-24 root(2 * 300), and two matrices' pairs of 2^-22, times |b| + 2 |c| = 9 and |X| = 1; each store at most half a step
    assert (got.double() - want.double()).norm() <= 9 * (2.0**-24 * 600**0.5 + 2 * 2.0**-22) + torch.finfo(dtype).eps * 1.01 * want.double().norm()
    assert torch.count_nonzero(g).item() <= few.numel()


def test_an_update_of_more_than_2_31_entries():
    m, n = 32800, 66000
    g = torch.randn((m, n), device="cuda")
    got = mats.orthogonalize(g, steps=1)
    x = g / g.double().norm().float()
    del g
    a = torch.matmul(x, x.t().contiguous())
    b = mats.QUINTIC[1] * a + mats.QUINTIC[2] * torch.matmul(a, a)
    for rows in (slice(0, 256), slice(m - 256, m)):
        want = mats.QUINTIC[0] * x[rows].double() + torch.matmul(b[rows], x).double()
        # fp32 products on both sides, of sums of up to 66000 terms: 2^-24 root(66000) each, four of them
        assert (got[rows].double() - want).norm() <= 8 * 2.0**-24 * 66000**0.5 * want.norm()
