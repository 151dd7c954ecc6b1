"""Matrices in four bits of include/qoda_matrices.h: rounding bit by bit, products and gradients against their formulas in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import matrix_definitions as M  # noqa: E402
import operator_definitions as D  # noqa: E402
from paper_2505_14371_amd import matrices as mats  # noqa: E402
from paper_2505_14371_amd import operators as ops  # noqa: E402
from test_gpu_operators import near, put  # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = list(ops.ACTIVATIONS)


@pytest.fixture(autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("a GPU test was selected but no GPU is visible")


def heavy(rng, *shape):
    return rng.standard_t(3, shape) * np.exp(rng.uniform(-6, 6, shape[:-1] + (1,)))


SIZES = [(1, 1), (1, 31), (2, 32), (3, 33), (37, 61), (64, 256), (65, 257), (63, 255), (130, 410), (1, 2048), (300, 8), (8, 300), (64, 511), (257, 96), (5, 4097)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_rounding(rows, cols, transposed, stochastic, dtype):
    rng = np.random.default_rng([rows, cols, transposed, stochastic])
    x, xd = put(heavy(rng, rows, cols), dtype, (0, 1, 8)[(rows + cols) % 3])
    seed, offset = 2**63 + 17, (3 << 32) + cols
    q = mats.microscale(x, transposed=transposed, rounding="stochastic" if stochastic else "nearest", seed=seed, offset=offset)
    want = M.mx(xd.T if transposed else xd, stochastic, seed, offset)
    codes, scales = M.laid_out(*want)
    assert q.shape == ((cols, rows) if transposed else (rows, cols))
    got = q.scales.cpu().numpy()
    assert got.shape == scales.shape and np.array_equal(got, scales), np.argwhere(got != scales)[:4]
    got = q.codes.cpu().numpy()
    assert got.shape == codes.shape and np.array_equal(got, codes), (np.argwhere(got != codes)[:4], got[got != codes][:4], codes[got != codes][:4])
    values = M.mx_values(*want)
    for t in TYPES.values():
        assert np.array_equal(q.values(t).double().cpu().numpy(), values)
    again = mats.Microscaled(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), *q.shape)
    assert np.array_equal(again.values().double().cpu().numpy(), values)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("stochastic", [False, True])
def test_every_scale_and_every_border(stochastic, transposed, dtype):
    """Blocks whose largest magnitude is each power of two (subnormal ones among them), just below and 1.5 times it, filled with the grid's
    places, the middles between them and their neighbours of the type."""
    t = TYPES[dtype]
    tiny = -149 if dtype == "f32" else -133
    top = np.array([m * 2.0**e for e in range(tiny, 128) for m in (1.0, 1.5, 1.99, 1.51)])
    top = np.unique(torch.from_numpy(top).to(t).double().numpy())
    top = top[(top > 0) & np.isfinite(top)]
    places = np.sort(np.concatenate([M.GRID, (M.GRID[:-1] + M.GRID[1:]) / 2]))[:15]
    unit = np.exp2(np.floor(np.log2(top)) - 2)
    body = np.concatenate([places, np.nextafter(places[1:].astype(np.float32), np.float32(0)), [-0.0]])
    v = torch.from_numpy(body[None, :] * unit[:, None]).to(t).double().numpy()
    v = np.clip(v, -top[:, None], top[:, None])
    v[:, 1::2] *= -1
    x = np.concatenate([v, top[:, None], np.zeros((len(top), 1))], axis=1)
    assert x.shape[1] == 32
    xt, xd = put(x.T if transposed else x, dtype)
    xd = xd.T if transposed else xd
    q = mats.microscale(xt, transposed=transposed, rounding="stochastic" if stochastic else "nearest", seed=5, offset=9)
    want = M.mx(xd, stochastic, 5, 9)
    codes, scales = M.laid_out(*want)
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    got = q.codes.cpu().numpy()
    off = np.argwhere((got != codes).any(1)).ravel()
    assert off.size == 0, (off[:4], top[off[:4]], got[off[0]], codes[off[0]])
    values = M.mx_values(*want)
    # from above 3 2^126 an entry may go to 4 2^126, which is 2^128 and no number of either type
    values[np.abs(values) >= 2.0**128] *= np.inf
    assert np.array_equal(q.values().double().cpu().numpy(), values)
    assert np.array_equal(q.values(torch.bfloat16).double().cpu().numpy(), values)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("stochastic", [False, True])
def test_infinities_and_nan_make_their_block_nan(stochastic, transposed, dtype):
    x = np.random.default_rng(3).standard_normal((70, 100))
    x[0, 0], x[3, 40], x[69, 99], x[5, 5] = np.inf, np.nan, -np.inf, -np.nan
    xt, xd = put(x.T if transposed else x, dtype)
    xd = xd.T if transposed else xd
    q = mats.microscale(xt, transposed=transposed, rounding="stochastic" if stochastic else "nearest", seed=5, offset=9)
    codes, scales = M.laid_out(*M.mx(xd, stochastic, 5, 9))
    assert np.array_equal(q.codes.cpu().numpy(), codes) and np.array_equal(q.scales.cpu().numpy(), scales)
    values = q.values(TYPES[dtype]).float().cpu().numpy()
    bad = np.zeros(x.shape, bool)
    bad[0, :32] = bad[3, 32:64] = bad[69, 96:] = bad[5, :32] = True
    assert np.array_equal(np.isnan(values), bad)
    w = mats.microscale(put(np.ones((5, 100)), dtype)[0])
    y = mats.mx_linear(q, w).float().cpu().numpy()               # tiles
    few = mats.mx_linear(q_rows(xd, slice(0, 6), dtype), w).float().cpu().numpy()
    assert np.array_equal(np.isnan(y).all(1), bad.any(1)) and np.array_equal(np.isnan(y).any(1), bad.any(1))
    assert np.array_equal(np.isnan(few).all(1), bad[:6].any(1)) and np.array_equal(np.isnan(few).any(1), bad[:6].any(1))


def q_rows(x, rows, dtype):
    return put(x[rows], dtype)[0]


def test_stochastic_rounding_keeps_the_mean():
    """The mean of n roundings of an entry is off by at most 2^-17 of the neighbours' distance d, and by five of its deviations, at most d / (2 root n)."""
    rng = np.random.default_rng(1)
    x, xd = put(rng.standard_normal((16, 64)))
    n = 1024
    total = torch.zeros_like(x, dtype=torch.float64)
    for k in range(n):
        total += mats.microscale(x, rounding="stochastic", seed=7, offset=k).values()
    _, e = M.mx(xd, True)
    unit = np.repeat(np.exp2(e.astype(float)), 32, axis=1)
    d = np.where(np.abs(xd) < 2 * unit, 0.5, np.where(np.abs(xd) < 4 * unit, 1.0, 2.0)) * unit
    assert (np.abs(total.cpu().numpy() / n - xd) <= d * (2.0**-17 + 5 * 0.5 / np.sqrt(n))).all()


def matrix(rng, rows, cols, dtype="f32", pad=0):
    """A microscaled matrix and what it stands for."""
    x, xd = put(heavy(rng, rows, cols) / max(1, cols) ** 0.5, dtype, pad)
    return mats.microscale(x), M.rounded(xd)


PRODUCTS = [(0, 5, 7), (5, 0, 7), (20, 0, 7), (5, 7, 0), (1, 1, 1), (1, 64, 256), (1, 513, 130), (2, 7, 3), (3, 33, 257), (5, 200, 410), (16, 64, 64), (17, 65, 33),
            (33, 410, 100), (64, 64, 128), (65, 129, 127), (127, 40, 129), (128, 256, 128), (130, 31, 258), (257, 96, 255), (256, 128, 256),
            (300, 520, 264), (513, 72, 520), (1024, 64, 8), (7, 2100, 410), (40, 4100, 24), (700, 24, 1000), (9, 300, 12000)]


@pytest.mark.parametrize("plain", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cin,cout", PRODUCTS)
def test_linear(rows, cin, cout, dtype, plain):
    rng = np.random.default_rng([rows, cin, cout])
    i = PRODUCTS.index((rows, cin, cout))
    a, p, pad = ACTS[i % 5], (0.0, 0.1, 0.5)[i % 3], (0, 1, 8)[(i // 2) % 3]
    x, xd = put(rng.standard_normal((rows, cin)), dtype, pad)
    xd = M.rounded(xd)
    w, wd = matrix(rng, cout, cin)
    b, bd = put(rng.standard_normal(cout))
    r, rd = put(rng.standard_normal((rows, cout)), dtype, pad)
    with_bias, with_res = i % 4 != 1, i % 2 == 0
    first = x if plain else mats.microscale(x)
    args = dict(activation=a, p=p, seed=11 + i, offset=(5 << 32) + i, dtype=None if plain else TYPES[dtype])
    y, z = mats.mx_linear(first, w, b if with_bias else None, r if with_res else None, keep_pre=True, **args)
    y1 = mats.mx_linear(first, w, b if with_bias else None, r if with_res else None, **args)
    assert y.shape == (rows, cout) and y.dtype == TYPES[dtype]
    wy, wz = D.linear(xd, wd, bd if with_bias else None, rd if with_res else None, a, p, 11 + i, (5 << 32) + i)
    bz = D.sum_bound(cin, np.abs(xd) @ np.abs(wd).T + np.abs(bd))
    near(z, wz, D.stored(bz, wz, dtype), "pre")
    scale = 2.0 if p == 0.5 else 1.2
    by = scale * (1.13 * bz + D.ACT_ERROR * (1 + np.abs(wz))) + 4 * D.U32 * (np.abs(wy) + np.abs(rd))
    near(y, wy, D.stored(by, wy, dtype), "y")
    assert torch.equal(y, y1)


@pytest.mark.parametrize("plain", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cin,cout", PRODUCTS)
def test_linear_input_grad(rows, cin, cout, dtype, plain):
    rng = np.random.default_rng([rows, cin, cout, 1])
    i = PRODUCTS.index((rows, cin, cout))
    a, p, pad = ACTS[(i + 2) % 5], (0.1, 0.0, 0.5)[i % 3], (0, 1, 8)[(i // 3) % 3]
    dz, dzd = put(heavy(rng, rows, cout), dtype, pad)
    dzd = M.rounded(dzd) if plain else M.rounded(dzd, True, 3, 77)
    w, wd = put(rng.standard_normal((cout, cin)) / np.sqrt(max(cout, 1)), dtype, pad)
    wtd = M.rounded(wd.T)
    z, zd = put(2 * rng.standard_normal((rows, cin)), dtype, pad)
    r, rd = put(rng.standard_normal((rows, cin)), dtype, pad)
    with_res, with_pre = i % 2 == 0, a != "none"
    first = dz if plain else mats.microscale(dz, rounding="stochastic", seed=3, offset=77)
    dx = mats.mx_linear_input_grad(first, mats.microscale(w, transposed=True), pre=z if with_pre else None, activation=a, p=p, seed=3, offset=i,
                                   residual=r if with_res else None, dtype=None if plain else TYPES[dtype])
    want = D.linear_input_grad(dzd, wtd.T, zd if with_pre else None, a, p, 3, i, rd if with_res else None)
    c = D.sum_bound(cout, np.abs(dzd) @ np.abs(wtd.T))
    scale = 2.0 if p == 0.5 else 1.2
    bound = scale * (1.13 * c + D.ACT_ERROR * (1 + np.abs(zd)) * np.abs(dzd @ wtd.T)) + 4 * D.U32 * (np.abs(want) + np.abs(rd))
    near(dx, want, D.stored(bound, want, dtype), "dx")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cin,cout", PRODUCTS)
def test_linear_weight_grad(rows, cin, cout, dtype):
    rng = np.random.default_rng([rows, cin, cout, 2])
    pad = (0, 1, 8)[PRODUCTS.index((rows, cin, cout)) % 3]
    dz, dzd = put(heavy(rng, rows, cout), dtype, pad)
    x, xd = put(rng.standard_normal((rows, cin)), dtype, pad)
    dzt, xt = mats.microscale(dz, transposed=True, rounding="stochastic", seed=1, offset=2), mats.microscale(x, transposed=True)
    dzd, xd = M.rounded(dzd.T, True, 1, 2), M.rounded(xd.T)
    dw, db = mats.mx_linear_weight_grad(dzt, xt)
    bw, bb = D.sum_bound(rows, np.abs(dzd) @ np.abs(xd).T), D.sum_bound(rows, np.abs(dzd).sum(1))
    near(dw, dzd @ xd.T, bw + 1e-38, "dw")
    near(db, dzd.sum(1), bb + 1e-38, "db")
    dw1, db1 = dw.clone(), db.clone()
    again = mats.mx_linear_weight_grad(dzt, xt, dw, db, accumulate=True)
    assert again[0] is dw and again[1] is db
    near(dw, 2 * dzd @ xd.T, 2 * bw + 2 * D.U32 * np.abs(2 * dzd @ xd.T) + 1e-38, "dw added")
    near(db, 2 * dzd.sum(1), 2 * bb + 2 * D.U32 * np.abs(2 * dzd.sum(1)) + 1e-38, "db added")
    only, none = mats.mx_linear_weight_grad(dzt, xt, bias=False)
    assert none is None and torch.equal(only, dw1)
    assert torch.equal(mats.mx_linear_weight_grad(dzt, xt)[1], db1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [16, 17, 100, 300])
def test_a_row_gives_the_same_alone_and_among_others(rows, dtype):
    """Sums of up to two steps have one order, whatever the tile."""
    rng = np.random.default_rng(rows)
    x, _ = put(rng.standard_normal((rows, 200)), dtype)
    w, _ = matrix(rng, 333, 200)
    whole = mats.mx_linear(x, w)
    assert torch.equal(mats.mx_linear(x[3], w), whole[3]) and torch.equal(mats.mx_linear(x[5:15], w), whole[5:15])
    assert torch.equal(mats.mx_linear(x.view(rows // 2, 2, 200), w).view(rows, -1), whole) if rows % 2 == 0 else True
    assert torch.equal(mats.mx_linear(mats.microscale(x), w, dtype=TYPES[dtype]), whole)


# the largest tiles with ragged ends on every side, and sums split along l; against 64-bit products on the GPU
LARGER = [(4000, 2100, 2300), (8190, 520, 4104), (600, 8200, 300), (30, 20000, 520), (2050, 1000, 6140), (100, 16000, 130)]


@pytest.mark.parametrize("rows,cin,cout", LARGER)
def test_larger(rows, cin, cout):
    gen = torch.Generator("cuda").manual_seed(rows)
    x, w, dz = (torch.randn(s, device="cuda", generator=gen) for s in ((rows, cin), (cout, cin), (rows, cout)))
    xq, wq, dzq = mats.microscale(x), mats.microscale(w), mats.microscale(dz)
    xt, wt, dzt = (mats.microscale(v, transposed=True) for v in (x, w, dz))
    for got, a, b, k in ((mats.mx_linear(xq, wq, dtype=torch.float32), xq, wq, cin), (mats.mx_linear_input_grad(dzq, wt, dtype=torch.float32), dzq, wt, cout),
                         (mats.mx_linear_weight_grad(dzt, xt)[0], dzt, xt, rows)):
        a, b = a.values().double(), b.values().double().t().contiguous()
        want, bound = torch.matmul(a, b), D.sum_bound(k, 1.0) * torch.matmul(a.abs(), b.abs())
        bad = ~((got.double() - want).abs() <= bound + want.abs() * 2.0**-24 + 1e-38)
        assert not bad.any(), (int(bad.sum()), bad.nonzero()[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_look_at_the_arguments_in_python_gives_the_same(monkeypatch, dtype):
    rng = np.random.default_rng(8)
    x, dz, r = (put(rng.standard_normal(s), dtype, 3)[0] for s in ((40, 300), (40, 70), (40, 70)))
    w, b, g = put(rng.standard_normal((70, 300)))[0], put(rng.standard_normal(70))[0], put(rng.standard_normal((2, 30, 50)), dtype, 2)[0]

    def everything():
        wq, wt, xq = mats.microscale(w), mats.microscale(w, transposed=True), mats.microscale(x, rounding="stochastic", seed=1, offset=2)
        dzt, xt = mats.microscale(dz, transposed=True), mats.microscale(x, transposed=True)
        out = [wq.codes, wq.scales, wt.codes, wt.scales, xq.values(), xq.values(torch.bfloat16)]
        out += mats.mx_linear(x, wq, b, r, activation="gelu", p=0.3, seed=4, offset=5, keep_pre=True)
        out += [mats.mx_linear(x.view(4, 10, 300) if x.is_contiguous() else x, wq), mats.mx_linear(xq, wq, dtype=torch.float32), mats.mx_linear(xq, wq), mats.mx_linear(x[7], wq)]
        out += [mats.mx_linear_input_grad(dz, wt, pre=x, activation="silu", p=0.2, seed=3, residual=x), mats.mx_linear_input_grad(mats.microscale(dz), wt, dtype=torch.bfloat16)]
        out += mats.mx_linear_weight_grad(dzt, xt)
        dw, db = torch.ones(70, 300, device="cuda"), torch.ones(70, device="cuda")
        out += mats.mx_linear_weight_grad(dzt, xt, dw, db, accumulate=True)
        out += [mats.mx_linear_weight_grad(dzt, xt, bias=False)[0], mats.orthogonalize(g), mats.orthogonalize(g, steps=2, out=torch.empty_like(g))]
        return out

    native = everything()
    assert mats._native is not None
    monkeypatch.setattr(mats, "_native", None)
    for a, c in zip(native, everything()):
        assert a.dtype == c.dtype and torch.equal(a, c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cin,cout", [(2, 2000, 30000), (16, 700, 90000), (9, 300, 40000)])
def test_few_rows_by_many(rows, cin, cout, dtype):
    """Rounded inside the product or before it, whichever takes less: the same."""
    gen = torch.Generator("cuda").manual_seed(rows)
    x, w = torch.randn(rows, cin, device="cuda", generator=gen).to(TYPES[dtype]), mats.microscale(torch.randn(cout, cin, device="cuda", generator=gen))
    y = mats.mx_linear(x, w)
    assert torch.equal(y, mats.mx_linear(mats.microscale(x), w, dtype=TYPES[dtype]))
    a, b = mats.microscale(x).values().double(), w.values().double().t().contiguous()
    want, bound = torch.matmul(a, b), D.sum_bound(cin, 1.0) * torch.matmul(a.abs(), b.abs())
    assert ((y.double() - want).abs() <= bound + (want.abs() + bound) * (D.STORE[dtype] * 1.001) + 1e-38).all()


@pytest.mark.parametrize("look", ["native", "python"])
def test_refusals(monkeypatch, look):
    mats._load()
    if look == "python":
        monkeypatch.setattr(mats, "_native", None)
    x, w = torch.randn(20, 64, device="cuda"), mats.microscale(torch.randn(32, 64, device="cuda"))
    q, r = mats.microscale(x), torch.randn(20, 32, device="cuda")
    for bad in (lambda: mats.microscale(x.half()), lambda: mats.microscale(x.t()), lambda: mats.microscale(x.cpu()), lambda: mats.microscale(x, rounding="down"),
                lambda: mats.microscale(x, seed=-1), lambda: mats.microscale(x, offset=1 << 64), lambda: mats.microscale(torch.tensor(1.0, device="cuda")), lambda: mats.microscale(3),
                lambda: mats.mx_linear(x[:, :40], w), lambda: mats.mx_linear(x, x), lambda: mats.mx_linear(q, w, residual=r), lambda: mats.mx_linear(x, w, dtype=torch.bfloat16),
                lambda: mats.mx_linear(q, w, dtype=torch.float16), lambda: mats.mx_linear(x, w, r), lambda: mats.mx_linear(x, w, activation="tanh"), lambda: mats.mx_linear(x, w, residual=r[:10]),
                lambda: mats.mx_linear(x, w, seed=-1), lambda: mats.mx_linear_input_grad(x, w, pre=r.bfloat16()), lambda: mats.mx_linear_input_grad(q, q.values()),
                lambda: mats.mx_linear_weight_grad(q, mats.microscale(x[:, :40])), lambda: mats.mx_linear_weight_grad(q, q, accumulate=True), lambda: mats.mx_linear_weight_grad(q, q, dweight=torch.empty(20, 64, device="cuda")),
                lambda: mats.mx_linear_weight_grad(q, q, dweight=torch.empty(20, 20)), lambda: mats.mx_linear_weight_grad(q, q, dbias=torch.empty(21, device="cuda")),
                lambda: q.values(torch.float64), lambda: mats.mx_linear(mats.Microscaled(q.codes.cpu(), q.scales.cpu(), 20, 64), w)):
        with pytest.raises(ValueError):
            bad()
    from paper_2505_14371_amd import qoda

    for bad in (lambda: mats.mx_linear(x, w, p=1.5), lambda: mats.mx_linear_input_grad(x, w, activation="relu")):
        with pytest.raises(qoda.QodaError):
            bad()
    x.requires_grad_()
    with pytest.raises(RuntimeError, match="no derivative"):
        mats.microscale(x)
    y = mats.mx_linear(x, w)
    assert y.requires_grad
    with pytest.raises(RuntimeError, match="records nothing"):
        y.sum().backward()
    with torch.no_grad():
        assert not mats.mx_linear(x, w).requires_grad and mats.microscale(x).shape == (20, 64)


def called(name, args):
    """A call of the C interface, its workspace full of NaN."""
    lib, stream = mats._load(), torch.cuda.current_stream().cuda_stream
    if name in ("mx_quantize", "mx_values"):
        assert getattr(lib, "qoda_" + name)(args, stream) == 0
        return
    need = getattr(lib, f"qoda_{name}_workspace_bytes")(args)
    assert need >= 0
    work = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda")
    assert getattr(lib, "qoda_" + name)(args, work.data_ptr() if need else None, need, stream) == 0
    assert (work[need:] == 255).all()


class Framed:
    """A matrix inside a larger one: rows `pad` entries further apart than they are long, and entries before and behind that are to stay what they are."""

    def __init__(self, rows, cols, dtype, pad):
        self.store = torch.full((rows * (cols + pad) + 40,), 7.0, dtype=dtype, device="cuda")
        self.t = self.store[pad: pad + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        self.at = (self.t.data_ptr(), cols + pad)

    def taken(self):
        got = self.t.clone()
        self.t.fill_(7.0)
        assert (self.store == 7.0).all()
        return got


@pytest.mark.parametrize("pad", [1, 3, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("plain", [True, False])
@pytest.mark.parametrize("rows,cin,cout", [(5, 300, 203), (70, 300, 203), (33, 8200, 61), (300, 260, 1030), (4000, 130, 2300)])
def test_through_the_c_interface(rows, cin, cout, plain, dtype, pad):
    """Outputs with strides of their own at any alignment, the residual in the output's memory, workspaces that hold anything."""
    gen = torch.Generator("cuda").manual_seed(rows)
    T, dt = TYPES[dtype], ops.DTYPES[TYPES[dtype]]
    x, z, r, dz = (torch.randn(s, device="cuda", generator=gen).to(T) for s in ((rows, cin), (rows, cin), (rows, cout), (rows, cout)))
    w, b = torch.randn((cout, cin), device="cuda", generator=gen), torch.randn(cout, device="cuda", generator=gen)
    wq, wt, xq, dzq, xt, dzt = (mats.microscale(v, transposed=t) for v, t in ((w, 0), (w, 1), (x, 0), (dz, 0), (x, 1), (dz, 1)))
    y, pre = Framed(rows, cout, T, pad), Framed(rows, cout, T, pad)
    y.t.copy_(r)
    called("mx_linear", mats._LINEAR.pack(dt, ops._number("gelu"), rows, cin, cout, *((x.data_ptr(), cin, 0, 0) if plain else (0, 0, *mats._mx(xq))), *mats._mx(wq), *y.at, *y.at, *pre.at,
                                          b.data_ptr(), 0.1, 3, 4))
    want, want_pre = mats.mx_linear(x if plain else xq, wq, b, r, activation="gelu", p=0.1, seed=3, offset=4, keep_pre=True, dtype=T)
    assert torch.equal(y.taken(), want) and torch.equal(pre.taken(), want_pre)
    dx = Framed(rows, cin, T, pad)
    dx.t.copy_(x)
    called("mx_linear_input_grad", mats._INPUT_GRAD.pack(dt, ops._number("silu"), rows, cin, cout, *((dz.data_ptr(), cout, 0, 0) if plain else (0, 0, *mats._mx(dzq))), *mats._mx(wt),
                                                         z.data_ptr(), cin, *dx.at, *dx.at, 0.1, 3, 4))
    assert torch.equal(dx.taken(), mats.mx_linear_input_grad(dz if plain else dzq, wt, pre=z, activation="silu", p=0.1, seed=3, offset=4, residual=x, dtype=T))
    dw, db = Framed(cout, cin, torch.float32, pad), Framed(1, cout, torch.float32, pad)
    dw.t.fill_(0.5), db.t.fill_(0.25)
    called("mx_linear_weight_grad", mats._WEIGHT_GRAD.pack(1, rows, cin, cout, *mats._mx(dzt), *mats._mx(xt), *dw.at, db.at[0]))
    want = mats.mx_linear_weight_grad(dzt, xt, torch.full((cout, cin), 0.5, device="cuda"), torch.full((cout,), 0.25, device="cuda"), accumulate=True)
    assert torch.equal(dw.taken(), want[0]) and torch.equal(db.taken()[0], want[1])
    v = Framed(rows, cin, T, pad)
    called("mx_values", mats._VALUES.pack(dt, rows, cin, *mats._mx(xq), *v.at))
    assert torch.equal(v.taken(), xq.values(T))
    v.t.copy_(x)
    for t in (0, 1):
        q = mats.microscale(x, transposed=t, rounding="stochastic", seed=5, offset=6)
        codes, scales = (torch.full((u.numel() + 64,), 99, dtype=torch.uint8, device="cuda") for u in (q.codes, q.scales))
        called("mx_quantize", mats._QUANTIZE.pack(dt, t, 1, rows, cin, *v.at, codes.data_ptr(), scales.data_ptr(), 5, 6))
        for got, u in ((codes, q.codes), (scales, q.scales)):
            assert torch.equal(got[:u.numel()], u.flatten()) and (got[u.numel():] == 99).all()
