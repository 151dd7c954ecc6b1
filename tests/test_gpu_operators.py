"""The matrix products, dropout and group normalisation of include/qoda_operators.h against their formulas in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import operator_definitions as D  # noqa: E402
from paper_2505_14371_amd import operators as ops  # noqa: E402
from paper_2505_14371_amd import qoda  # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = list(ops.ACTIVATIONS)


@pytest.fixture(autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("a GPU test was selected but no GPU is visible")


def put(a, dtype="f32", pad=0):
    """A tensor of this type on the GPU with rows ``pad`` entries further apart, what is between them NaN; and its values in 64 bits."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(TYPES[dtype])
    wide = torch.full(t.shape[:-1] + (t.shape[-1] + pad,), float("nan"), dtype=TYPES[dtype])
    wide[..., : t.shape[-1]] = t
    return wide.cuda()[..., : t.shape[-1]], t.double().numpy()


def near(got, want, bound, what):
    got = got.double().cpu().numpy().reshape(want.shape)
    bad = ~(np.abs(got - want) <= bound)
    if bad.any():
        pytest.fail(f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}, bound {np.broadcast_to(bound, want.shape)[bad][0]}")


# sizes: empty, single, around the multiples of 8, 16, 32, 64, 128 and 256 that tiles, lanes and blocks of lots have, odd widths
# of the workloads, and shapes with one long side
PRODUCTS = [(0, 5, 7), (5, 0, 7), (5, 7, 0), (1, 1, 1), (1, 64, 256), (1, 513, 130), (2, 7, 3), (3, 33, 257), (5, 200, 410), (16, 64, 64), (17, 65, 33),
            (33, 410, 100), (64, 64, 128), (65, 129, 127), (127, 40, 129), (128, 256, 128), (130, 31, 258), (257, 96, 255), (256, 128, 256),
            (300, 520, 264), (513, 72, 520), (1024, 64, 8), (7, 2100, 410), (40, 4100, 24), (700, 24, 1000)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cin,cout", PRODUCTS)
def test_linear(rows, cin, cout, dtype):
    rng = np.random.default_rng([rows, cin, cout])
    i = PRODUCTS.index((rows, cin, cout))
    a, p, pad = ACTS[i % 5], (0.0, 0.1, 0.5)[i % 3], (0, 1, 8)[(i // 2) % 3]
    x, xd = put(rng.standard_normal((rows, cin)), dtype, pad)
    w, wd = put(rng.standard_normal((cout, cin)) / np.sqrt(max(cin, 1)), dtype, pad)
    b, bd = put(rng.standard_normal(cout))
    r, rd = put(rng.standard_normal((rows, cout)), dtype, pad)
    with_bias, with_res = i % 4 != 1, i % 2 == 0
    y, z = ops.linear(x, w, b if with_bias else None, r if with_res else None, activation=a, p=p, seed=11 + i, offset=(5 << 32) + i, keep_pre=True)
    y1 = ops.linear(x, w, b if with_bias else None, r if with_res else None, activation=a, p=p, seed=11 + i, offset=(5 << 32) + i)
    wy, wz = D.linear(xd, wd, bd if with_bias else None, rd if with_res else None, a, p, 11 + i, (5 << 32) + i)
    bz = D.sum_bound(cin, np.abs(xd) @ np.abs(wd).T + np.abs(bd))
    near(z, wz, D.stored(bz, wz, dtype), "pre")
    scale = 2.0 if p == 0.5 else 1.2
    by = scale * (1.13 * bz + D.ACT_ERROR * (1 + np.abs(wz))) + 4 * D.U32 * (np.abs(wy) + np.abs(rd))
    near(y, wy, D.stored(by, wy, dtype), "y")
    assert torch.equal(y, y1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cin,cout", PRODUCTS)
def test_linear_input_grad(rows, cin, cout, dtype):
    rng = np.random.default_rng([rows, cin, cout, 1])
    i = PRODUCTS.index((rows, cin, cout))
    a, p, pad = ACTS[(i + 2) % 5], (0.1, 0.0, 0.5)[i % 3], (0, 1, 8)[(i // 3) % 3]
    dz, dzd = put(rng.standard_normal((rows, cout)), dtype, pad)
    w, wd = put(rng.standard_normal((cout, cin)) / np.sqrt(max(cout, 1)), dtype, pad)
    z, zd = put(2 * rng.standard_normal((rows, cin)), dtype, pad)
    r, rd = put(rng.standard_normal((rows, cin)), dtype, pad)
    with_res, with_pre = i % 2 == 0, a != "none"
    dx = ops.linear_input_grad(dz, w, pre=z if with_pre else None, activation=a, p=p, seed=3, offset=i, residual=r if with_res else None)
    want = D.linear_input_grad(dzd, wd, zd if with_pre else None, a, p, 3, i, rd if with_res else None)
    c = D.sum_bound(cout, np.abs(dzd) @ np.abs(wd))
    scale = 2.0 if p == 0.5 else 1.2
    bound = scale * (1.13 * c + D.ACT_ERROR * (1 + np.abs(zd)) * np.abs(dzd @ wd)) + 4 * D.U32 * (np.abs(want) + np.abs(rd))
    near(dx, want, D.stored(bound, want, dtype), "dx")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cin,cout", PRODUCTS)
def test_linear_weight_grad(rows, cin, cout, dtype):
    rng = np.random.default_rng([rows, cin, cout, 2])
    pad = (0, 1, 8)[PRODUCTS.index((rows, cin, cout)) % 3]
    dz, dzd = put(rng.standard_normal((rows, cout)), dtype, pad)
    x, xd = put(rng.standard_normal((rows, cin)), dtype, pad)
    dw, db = ops.linear_weight_grad(dz, x)
    bw, bb = D.sum_bound(rows, np.abs(dzd).T @ np.abs(xd)), D.sum_bound(rows, np.abs(dzd).sum(0))
    near(dw, dzd.T @ xd, bw + 1e-38, "dw")
    near(db, dzd.sum(0), bb + 1e-38, "db")
    dw1, db1 = dw.clone(), db.clone()
    again = ops.linear_weight_grad(dz, x, dw, db, accumulate=True)
    assert again[0] is dw and again[1] is db
    near(dw, 2 * dzd.T @ xd, 2 * bw + 2 * D.U32 * np.abs(2 * dzd.T @ xd) + 1e-38, "dw added")
    near(db, 2 * dzd.sum(0), 2 * bb + 2 * D.U32 * np.abs(2 * dzd.sum(0)) + 1e-38, "db added")
    only, none = ops.linear_weight_grad(dz, x, bias=False)
    assert none is None and torch.equal(only, dw1)
    assert torch.equal(ops.linear_weight_grad(dz, x)[1], db1)


# what small products do not reach: the largest tiles with ragged ends on every side, sums split along l, rows at 4-byte and at odd addresses
LARGER = [(8190, 536, 8184, 0, "bf16"), (8184, 8184, 600, 0, "bf16"), (3000, 410, 2100, 0, "bf16"), (1500, 411, 1001, 0, "bf16"), (616, 8184, 8184, 0, "bf16"), (2000, 2040, 6136, 0, "bf16"), (6140, 2002, 2042, 2, "bf16"), (200, 8200, 300, 0, "bf16"), (30, 4104, 520, 0, "bf16"),
          (24, 5001, 333, 1, "bf16"), (3000, 410, 2100, 0, "f32"), (100, 6000, 130, 1, "f32"), (2050, 200, 2060, 0, "f32"), (20, 2000, 700, 0, "f32")]


def near64(got, want, bound, dtype, what):
    bound = bound + (want.abs() + bound) * (D.STORE[dtype] * 1.001) + 1e-38
    bad = ~((got.double() - want).abs() <= bound)
    if bad.any():
        at = tuple(int(v) for v in bad.nonzero()[0])
        pytest.fail(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {at}: {float(got[at])} for {float(want[at])}, bound {float(bound[at])}")


@pytest.mark.parametrize("rows,cin,cout,pad,dtype", LARGER)
def test_larger_products(rows, cin, cout, pad, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows + cin)

    def matrix(r, c, scale=1.0):
        wide = torch.full((r, c + pad), float("nan"), device="cuda", dtype=TYPES[dtype])
        wide[:, :c] = torch.randn((r, c), device="cuda", generator=gen) * scale
        return wide[:, :c]

    x, w, dz, r = matrix(rows, cin), matrix(cout, cin, cin ** -0.5), matrix(rows, cout), matrix(rows, cout)
    X, W, Z, R = (t.double().contiguous() for t in (x, w, dz, r))
    want, size = X @ W.t().contiguous(), X.abs() @ W.abs().t().contiguous()
    y, pre = ops.linear(x, w, residual=r, activation="relu", keep_pre=True)
    near64(pre, want, 2 * (cin + 4) * D.U32 * size, dtype, "pre")
    near64(y, R + want.clamp(min=0), 2 * (cin + 4) * D.U32 * size + 4 * D.U32 * (R.abs() + want.abs()), dtype, "y")
    want, size = Z @ W, Z.abs() @ W.abs()
    near64(ops.linear_input_grad(dz, w), want, 2 * (cout + 4) * D.U32 * size, dtype, "dx")
    want = torch.where(X > 0, want, torch.zeros_like(want)) + X
    near64(ops.linear_input_grad(dz, w, pre=x, activation="relu", residual=x), want, 2 * (cout + 4) * D.U32 * size + 4 * D.U32 * (size + X.abs()), dtype, "dx through relu")
    Zt = Z.t().contiguous()
    want, size = Zt @ X, Zt.abs() @ X.abs()
    dw, db = ops.linear_weight_grad(dz, x)
    near64(dw, want, 2 * (rows + 4) * D.U32 * size, "f32", "dw")
    near64(db, Z.sum(0), 2 * (rows + 4) * D.U32 * Z.abs().sum(0), "f32", "db")
    again = ops.linear_weight_grad(dz, x, dw.clone(), db.clone(), accumulate=True)
    near64(again[0], 2 * want, 4 * (rows + 4) * D.U32 * size, "f32", "dw added")
    near64(again[1], 2 * Z.sum(0), 4 * (rows + 4) * D.U32 * Z.abs().sum(0), "f32", "db added")
    assert torch.equal(ops.linear(x, w, residual=r, activation="relu"), y) and torch.equal(ops.linear_weight_grad(dz, x)[0], dw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cin,cout", [(7, 40, 33), (300, 200, 410), (20, 4000, 300), (130, 6000, 70)])
def test_a_residual_may_be_the_outputs_memory(rows, cin, cout, dtype):
    lib, dt = ops._load(), ops.DTYPES[TYPES[dtype]]
    x, w, r = (torch.randn(s, device="cuda").to(TYPES[dtype]) for s in ((rows, cin), (cout, cin), (rows, cout)))
    place = lambda t: (t.data_ptr(), t.shape[-1])  # noqa: E731

    def call(name, pack, *args):
        a = pack.pack(dt, *args)
        need = getattr(lib, f"qoda_{name}_workspace_bytes")(a)
        scratch = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        assert getattr(lib, f"qoda_{name}")(a, scratch.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == qoda.OK, ops.operator_error()

    y = r.clone()
    call("linear", ops._LINEAR, 3, rows, cin, cout, *place(x), *place(w), *place(y), *place(y), 0, 0, 0, 0.1, 1, 2)
    assert torch.equal(y, ops.linear(x, w, residual=r, activation="gelu", p=0.1, seed=1, offset=2))
    dx = x.clone()
    call("linear_input_grad", ops._INPUT_GRAD, 0, rows, cin, cout, *place(r), *place(w), 0, 0, *place(dx), *place(dx), 0.1, 1, 2)
    assert torch.equal(dx, ops.linear_input_grad(r, w, residual=x, p=0.1, seed=1, offset=2))
    for both in (False, True):
        y = r.clone()
        a = ops._DROPOUT.pack(dt, 1, rows, cout, *place(y), *place(y if both else r), *place(y), 0.5, 3, 4)
        assert lib.qoda_dropout(a, torch.cuda.current_stream().cuda_stream) == qoda.OK
        assert torch.equal(y, ops.dropout(r, 0.5, 3, 4, activation="relu", residual=r))
    n, mean, rstd = ops.group_norm(r, 1)
    want = ops.group_norm_grad(n, r, mean, rstd, 1, residual=r)
    dx, dw, db = r.clone(), torch.empty(cout, device="cuda"), torch.empty(cout, device="cuda")
    three = lambda t: (t.data_ptr(), t.shape[-1], t.shape[-1])  # noqa: E731
    call("group_norm_grad", ops._NORM_GRAD, 0, rows, 1, cout, 1, *three(n), *three(r), *three(dx), *three(dx), 0, 0, mean.data_ptr(), rstd.data_ptr(), dw.data_ptr(), db.data_ptr(), 0)
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1]) and torch.equal(db, want[2])


def test_a_workspace_that_is_too_small_is_refused():
    x, w = torch.randn((20, 4000), device="cuda"), torch.randn((300, 4000), device="cuda")
    y, lib = torch.zeros((20, 300), device="cuda"), ops._load()
    a = ops._LINEAR.pack(0, 0, 20, 4000, 300, x.data_ptr(), 4000, w.data_ptr(), 4000, 0, 0, y.data_ptr(), 300, 0, 0, 0, 0.0, 0, 0)
    need = lib.qoda_linear_workspace_bytes(a)
    assert need > 0
    scratch = torch.empty(need + 16, dtype=torch.uint8, device="cuda")
    for p, n, said in ((None, 0, "workspace"), (scratch.data_ptr(), need - 1, "workspace"), (scratch.data_ptr() + 4, need, "16 bytes")):
        assert lib.qoda_linear(a, p, n, None) == qoda.EINVAL and said in ops.operator_error()
    torch.cuda.synchronize()
    assert not y.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("activation", ACTS)
@pytest.mark.parametrize("rows,cols,pad", [(0, 4, 0), (3, 0, 0), (1, 1, 0), (1, 4099, 0), (7, 8, 0), (5, 61, 0), (5, 61, 1), (33, 410, 6), (64, 256, 8), (300, 1031, 1)])
def test_dropout_and_its_gradient(rows, cols, pad, activation, dtype):
    rng = np.random.default_rng([rows, cols, pad])
    x, xd = put(2 * rng.standard_normal((rows, cols)), dtype, pad)
    r, rd = put(rng.standard_normal((rows, cols)), dtype, pad)
    for p in (0.0, 0.1, 0.75, 1.0):
        scale = 1 / (1 - p) if p < 1 else 0.0
        want = D.drop(D.act(xd, activation), p, 2**63 + 5, 77)
        bound = 1.01 * scale * D.ACT_ERROR * (1 + np.abs(xd)) + 4 * D.U32 * np.abs(want)
        y = ops.dropout(x, p, 2**63 + 5, 77, activation=activation)
        near(y, want, D.stored(bound, want, dtype), f"y, p = {p}")
        if rows and cols:
            assert np.array_equal(y.double().cpu().numpy()[want == 0], want[want == 0])
        want_r = rd + want
        near(ops.dropout(x, p, 2**63 + 5, 77, activation=activation, residual=r), want_r, D.stored(bound + 2 * D.U32 * np.abs(want_r), want_r, dtype), "with residual")
        want_g = D.drop(rd * D.slope(xd, activation), p, 2**63 + 5, 77)
        bound = 1.01 * scale * D.ACT_ERROR * (1 + np.abs(xd)) * np.abs(rd) + 4 * D.U32 * np.abs(want_g)
        g = ops.dropout_grad(r, p, 2**63 + 5, 77, pre=None if activation == "none" else x, activation=activation)
        near(g, want_g, D.stored(bound, want_g, dtype), f"gradient, p = {p}")


def test_dropped_entries_are_zero_whatever_they_were():
    x = torch.full((40, 100), float("nan"), device="cuda")
    x[::2] = float("inf")
    pre = torch.full((40, 100), float("nan"), device="cuda")
    dropped = torch.from_numpy(D.lots(40, 100, 9, 1) < D.threshold(0.5)).cuda()
    for y in (ops.dropout(x, 0.5, 9, 1), ops.dropout_grad(x, 0.5, 9, 1, pre=pre, activation="gelu")):
        assert torch.equal(y[dropped], torch.zeros_like(y[dropped])) and not torch.isfinite(y[~dropped]).any()
    assert torch.equal(ops.dropout(x, 1.0, 9, 1), torch.zeros_like(x))
    w = torch.ones((100, 4), device="cuda")
    y = ops.linear(torch.full((40, 4), float("inf"), device="cuda"), w, p=0.5, seed=9, offset=1)
    assert torch.equal(y[dropped], torch.zeros_like(y[dropped])) and torch.isinf(y[~dropped]).all()


def test_a_value_that_is_not_finite_stays_in_its_row_and_column():
    """Rows and columns at a tile's edge are filled from nowhere else."""
    for dtype in TYPES:
        for rows, cin, cout in ((70, 61, 75), (1, 410, 70), (300, 130, 290)):
            x = torch.randn((rows, cin + 1), device="cuda").to(TYPES[dtype])
            x[:, -1] = float("nan")                           # next to every row's end
            w = torch.randn((cout, cin + 1), device="cuda").to(TYPES[dtype])
            w[:, -1] = float("inf")
            x, w = x[:, :cin], w[:, :cin]
            assert torch.isfinite(ops.linear(x, w)).all()
            dz = torch.randn((rows, cout + 1), device="cuda").to(TYPES[dtype])
            dz[:, -1] = float("nan")
            assert torch.isfinite(ops.linear_input_grad(dz[:, :cout], w)).all()
            dw, db = ops.linear_weight_grad(dz[:, :cout], x)
            assert torch.isfinite(dw).all() and torch.isfinite(db).all()
            x = x.clone()
            x[rows // 2, cin // 2] = float("inf")
            y = ops.linear(x, w)
            assert not torch.isfinite(y[rows // 2]).any() and torch.isfinite(y[: rows // 2]).all() and torch.isfinite(y[rows // 2 + 1:]).all()


NORMS = [(1, 1, 1, 1), (3, 1, 2, 1), (5, 1, 410, 1), (4, 1, 2048, 1), (2, 1, 8192, 1), (3, 1, 16391, 1), (1000, 1, 16, 1), (2, 9, 6, 3), (3, 16, 32, 8), (2, 256, 64, 32),
         (1, 1023, 24, 2), (5, 33, 70, 1), (2, 4, 96, 96), (3, 100, 130, 13), (1, 5000, 8, 1), (7, 64, 512, 16), (2, 1, 64, 8), (2, 1024, 64, 16), (1, 5000, 64, 2),
         (2, 3, 4100, 1), (1, 40, 5000, 2), (3, 1, 4100, 2), (2, 7, 264, 24), (1, 3000, 26, 2), (9000, 3, 8, 2), (2100, 5, 20, 4), (2048, 9, 24, 3), (2500, 30, 40, 5), (2200, 2, 600, 2), (0, 4, 8, 2), (3, 0, 8, 2), (2, 3, 0, 1)]


def norm_inputs(n, s, c, dtype, seed):
    rng = np.random.default_rng([n, s, c, seed])
    x, xd = put(rng.standard_normal((n, s, c)) * (0.5 + np.abs(rng.standard_normal(c))) + 3 * rng.standard_normal(c), dtype)
    w, wd = put(1 + 0.2 * rng.standard_normal(c))
    b, bd = put(0.2 * rng.standard_normal(c))
    return rng, x, xd, w, wd, b, bd


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,s,c,groups", NORMS)
def test_group_norm(n, s, c, groups, dtype):
    _, x, xd, w, wd, b, bd = norm_inputs(n, s, c, dtype, 0)
    a = ACTS[NORMS.index((n, s, c, groups)) % 5]
    y, mean, rstd = ops.group_norm(x, groups, w, b, activation=a)
    assert y.shape == x.shape and mean.shape == rstd.shape == (n, groups)
    if n * s * c == 0:
        return
    want, wm, wr, h, z = D.group_norm(xd, groups, wd, bd, 1e-5, a)
    k = s * c // groups
    # a mean of k terms; the squares about it; both from fp32 sums
    big = np.abs(xd).max()
    em = D.sum_bound(k, big)
    near(mean, wm, em + D.U32 * np.abs(wm), "mean")
    var = 1 / wr**2
    er = wr * (0.5 * (D.sum_bound(k, var) + em**2) / var + 4 * D.U32)
    near(rstd, wr, er, "rstd")
    wide = lambda v: np.repeat(v, c // groups, axis=1)[:, None, :]  # noqa: E731
    eh = (em + 2 * D.U32 * np.abs(xd)) * wide(wr) + np.abs(h) * wide(er / wr) + 2 * D.U32 * np.abs(h)
    bound = 1.13 * (eh * np.abs(wd) + 2 * D.U32 * np.abs(z)) + D.ACT_ERROR * (1 + np.abs(z))
    near(y, want, D.stored(bound, want, dtype), "y")
    y2, m2, r2 = ops.group_norm(x, groups, w, b, activation=a)
    assert torch.equal(y, y2) and torch.equal(mean, m2) and torch.equal(rstd, r2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,s,c,groups", NORMS)
def test_group_norm_grad(n, s, c, groups, dtype):
    rng, x, xd, w, wd, b, bd = norm_inputs(n, s, c, dtype, 1)
    i = NORMS.index((n, s, c, groups))
    a = ("none", "gelu", "silu")[i % 3]
    dy, dyd = put(rng.standard_normal((n, s, c)), dtype)
    r, rd = put(rng.standard_normal((n, s, c)), dtype)
    if n * s * c:
        _, wm, wr, _, _ = D.group_norm(xd, groups, wd, bd, 1e-5, a)
    else:
        wm, wr = np.zeros((n, groups)), np.ones((n, groups))
    mean, meand = put(wm)
    rstd, rstdd = put(wr)
    dx, dw, db = ops.group_norm_grad(dy, x, mean, rstd, groups, w, b, activation=a, residual=r if i % 2 else None)
    if n * s * c == 0:
        assert not dw.any() and not db.any()
        return
    want, wdw, wdb, u = D.group_norm_grad(dyd, xd, meand, rstdd, groups, wd, bd, a)
    wide = lambda v: np.repeat(v, c // groups, axis=1)[:, None, :]  # noqa: E731
    h = (xd - wide(meand)) * wide(rstdd)
    eh = 2 * D.U32 * (np.abs(xd) + np.abs(wide(meand))) * wide(rstdd) + 2 * D.U32 * np.abs(h)
    # the slope's own slope is below 1.1 everywhere; dh = dy * slope
    edh = np.abs(dyd) * (D.ACT_ERROR * (1 + np.abs(h * wd + bd)) + 1.2 * (eh * np.abs(wd) + 2 * D.U32 * (np.abs(h * wd) + np.abs(bd)))) + 2 * D.U32 * np.abs(dyd) * 1.13
    dh = np.abs(dyd) * 1.13
    four = lambda v: v.reshape(n, s, groups, c // groups)  # noqa: E731
    per = lambda v: np.broadcast_to(four(v).mean(axis=(1, 3), keepdims=True), four(v).shape).reshape(n, s, c)  # noqa: E731
    k = s * c // groups
    eu = edh * np.abs(wd) + 2 * D.U32 * dh * np.abs(wd)
    e1 = per(eu) + D.sum_bound(k, per(dh * np.abs(wd)))
    e2 = per(eu * np.abs(h) + dh * np.abs(wd) * eh) + D.sum_bound(k, per(dh * np.abs(wd) * np.abs(h)))
    m2 = np.abs(per(u * h))
    bound = wide(rstdd) * (eu + e1 + np.abs(h) * e2 + eh * m2 + 4 * D.U32 * (np.abs(u) + np.abs(per(u)) + np.abs(h) * m2))
    full = want + rd if i % 2 else want
    near(dx, full, D.stored(bound + 2 * D.U32 * np.abs(full), full, dtype), "dx")
    near(dw, wdw, D.sum_bound(n * s, (dh * np.abs(h)).sum((0, 1))) + (edh * np.abs(h) + dh * eh).sum((0, 1)), "dweight")
    near(db, wdb, D.sum_bound(n * s, dh.sum((0, 1))) + edh.sum((0, 1)), "dbias")
    dw1, db1 = dw.clone(), db.clone()
    dx2, dw2, db2 = ops.group_norm_grad(dy, x, mean, rstd, groups, w, b, activation=a, residual=r if i % 2 else None, dweight=dw, dbias=db, accumulate=True)
    assert torch.equal(dx, dx2) and dw2 is dw and db2 is db
    near(dw, 2 * dw1.double().cpu().numpy(), 2 * D.U32 * np.abs(2 * wdw) + 1e-38 + 4 * D.U32 * np.abs(wdw).max(), "dweight added")
    near(db, 2 * db1.double().cpu().numpy(), 2 * D.U32 * np.abs(2 * wdb) + 1e-38 + 4 * D.U32 * np.abs(wdb).max(), "dbias added")


def test_group_norm_of_strided_values_without_weights():
    wide = torch.randn((4, 6, 40), device="cuda")
    x = wide[:, ::2, 3:27]                                # positions two apart, channels inside a wider row
    y, mean, rstd = ops.group_norm(x, 3)
    z, m, r = ops.group_norm(x.contiguous(), 3)
    assert torch.equal(y, z) and torch.equal(mean, m) and torch.equal(rstd, r)
    g = ops.group_norm_grad(x, x, mean, rstd, 3)
    h = ops.group_norm_grad(x.contiguous(), x.contiguous(), mean, rstd, 3)
    assert all(torch.equal(a, b) for a, b in zip(g, h))
    maps = torch.randn((2, 5, 7, 16), device="cuda")      # [samples, height, width, channels]
    assert torch.equal(ops.group_norm(maps, 4)[0].view(2, 35, 16), ops.group_norm(maps.view(2, 35, 16), 4)[0])


def test_a_constant_and_a_far_mean_are_normalised():
    """The variance is that of the values about their mean, not a difference of large sums."""
    for dtype, far in (("f32", 4096.0), ("bf16", 128.0)):
        for shape, groups in (((8, 1, 2048), 1), ((2, 300, 32), 4), ((2, 5000, 64), 2)):
            x, xd = put(far + np.random.default_rng(1).standard_normal(shape), dtype)
            y, mean, rstd = ops.group_norm(x, groups)
            _, wm, wr, _, _ = D.group_norm(xd, groups, 1.0, 0.0, 1e-5, "none")
            assert np.abs(mean.double().cpu().numpy() - wm).max() <= 2e-6 * far
            assert np.abs(rstd.double().cpu().numpy() / wr - 1).max() <= 1e-4
            y, _, rstd = ops.group_norm(torch.full(shape, far, dtype=TYPES[dtype], device="cuda"), groups)
            assert not y.any() and torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5))


def differences(f, at, h=1e-6):
    """The gradient of a number f by central differences in 64 bits."""
    g = np.zeros_like(at)
    for i in np.ndindex(at.shape):
        up, down = at.copy(), at.copy()
        up[i] += h
        down[i] -= h
        g[i] = (f(up) - f(down)) / (2 * h)
    return g


@pytest.mark.parametrize("activation", ACTS)
def test_gradients_against_differences(activation):
    rng = np.random.default_rng(ACTS.index(activation))
    x, xd = put(rng.standard_normal((6, 9)))
    w1, w1d = put(rng.standard_normal((11, 9)) / 3)
    b1, b1d = put(rng.standard_normal(11))
    w2, w2d = put(rng.standard_normal((9, 11)) / 3)
    t, td = put(rng.standard_normal((6, 9)))

    def loss(x, w1, b1, w2):          # <t, x + drop(w2 drop(act(w1 x + b1)))>
        hid, _ = D.linear(x, w1, b1, None, activation, 0.25, 5, 1)
        y, _ = D.linear(hid, w2, None, x, "none", 0.25, 5, 2)
        return float((y * td).sum())

    hid, z = ops.linear(x, w1, b1, activation=activation, p=0.25, seed=5, offset=1, keep_pre=True)
    dz2 = ops.dropout_grad(t, 0.25, 5, 2)
    dw2, _ = ops.linear_weight_grad(dz2, hid)
    dz1 = ops.linear_input_grad(dz2, w2, pre=z, activation=activation, p=0.25, seed=5, offset=1)
    dw1, db1 = ops.linear_weight_grad(dz1, x)
    dx = ops.linear_input_grad(dz1, w1, residual=t)
    for got, want in ((dx, differences(lambda v: loss(v, w1d, b1d, w2d), xd)), (dw1, differences(lambda v: loss(xd, v, b1d, w2d), w1d)),
                      (db1, differences(lambda v: loss(xd, w1d, v, w2d), b1d)), (dw2, differences(lambda v: loss(xd, w1d, b1d, v), w2d))):
        # a difference is good to about 1e-9 of the loss, the fp32 chain to a few units of sums of at most 11 terms
        assert np.abs(got.double().cpu().numpy() - want).max() <= 1e-5 * (1 + np.abs(want).max())


@pytest.mark.parametrize("activation", ["none", "gelu", "silu"])
def test_group_norm_gradients_against_differences(activation):
    rng = np.random.default_rng(3)
    x, xd = put(rng.standard_normal((2, 3, 8)))
    w, wd = put(1 + 0.2 * rng.standard_normal(8))
    b, bd = put(0.2 * rng.standard_normal(8))
    t, td = put(rng.standard_normal((2, 3, 8)))
    loss = lambda x, w, b: float((D.group_norm(x, 2, w, b, 1e-5, activation)[0] * td).sum())  # noqa: E731
    _, mean, rstd = ops.group_norm(x, 2, w, b, activation=activation)
    dx, dw, db = ops.group_norm_grad(t, x, mean, rstd, 2, w, b, activation=activation)
    for got, want in ((dx, differences(lambda v: loss(v, wd, bd), xd)), (dw, differences(lambda v: loss(xd, v, bd), wd)), (db, differences(lambda v: loss(xd, wd, v), bd))):
        assert np.abs(got.double().cpu().numpy() - want).max() <= 1e-5 * (1 + np.abs(want).max())


def test_more_dimensions_are_rows():
    x, w = torch.randn((2, 3, 5, 16), device="cuda"), torch.randn((24, 16), device="cuda")
    y = ops.linear(x, w)
    assert y.shape == (2, 3, 5, 24) and torch.equal(y.view(30, 24), ops.linear(x.view(30, 16), w))
    v = torch.randn(16, device="cuda")
    assert torch.equal(ops.linear(v, w), ops.linear(v.view(1, 16), w).view(24))
    assert torch.equal(ops.dropout(x, 0.3, 1, 2).view(30, 16), ops.dropout(x.view(30, 16), 0.3, 1, 2))


def test_offsets_beyond_32_bits():
    """Matrices of more than 2^31 entries and of more than 4 GB: the last rows are right, and their lots are of their own rows."""
    rows, cols = 65600, 32776
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    tail = torch.randn((64, cols), device="cuda").to(torch.bfloat16)
    x.zero_()
    x[-64:] = tail
    y = ops.dropout(x, 0.25, 3, 4)
    want = D.drop(tail.double().cpu().numpy(), 0.25, 3, 4, first_row=rows - 64)
    near(y[-64:], want, D.stored(np.abs(want) * 4 * D.U32, want, "bf16"), "the last rows")
    assert not y[:64].any()
    del y
    w = (torch.randn((24, cols), device="cuda") / 181).to(torch.bfloat16)
    z = ops.linear(x, w)
    assert torch.equal(z[-64:], ops.linear(tail, w)) or torch.allclose(z[-64:].float(), ops.linear(tail, w).float(), rtol=2**-7, atol=1e-3)
    assert not z[: rows - 64].any()
    y, mean, rstd = ops.group_norm(x, 1)
    y2, mean2, rstd2 = ops.group_norm(tail, 1)
    assert torch.equal(y[-64:], y2) and torch.equal(mean[-64:], mean2)


def test_runs_on_the_stream_it_is_given():
    x, w = torch.randn((500, 300), device="cuda"), torch.randn((200, 300), device="cuda")
    want = ops.linear(x, w, activation="silu")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    big = torch.randn((4000, 4000), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        late = torch.zeros_like(x)
        for _ in range(20):
            big = big @ big * 1e-4
        late.copy_(x)                                   # behind the products on s
    got = ops.linear(late, w, activation="silu", stream=s)
    handle = ops.linear(late, w, activation="silu", stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(got, want) and torch.equal(handle, want)


def test_captured_calls_replay():
    x, w, b = torch.randn((130, 96), device="cuda"), torch.randn((70, 96), device="cuda"), torch.randn(70, device="cuda")
    scale, shift = torch.rand(70, device="cuda"), torch.rand(70, device="cuda")

    def work():
        y, z = ops.linear(x, w, b, activation="gelu", p=0.1, seed=1, offset=2, keep_pre=True)
        n, mean, rstd = ops.group_norm(y, 1, scale, shift)
        dn, dscale, dshift = ops.group_norm_grad(n, y, mean, rstd, 1, scale, shift)
        dz = ops.dropout_grad(dn, 0.1, 1, 2, pre=z, activation="gelu")
        dw, db = ops.linear_weight_grad(dz, x)
        return [n, dscale, dshift, dz, dw, db, ops.linear_input_grad(dz, w, residual=x)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work()
    for k in range(4):
        x.copy_(torch.randn((130, 96), device="cuda") * (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        want = work()
        for a, c in zip(got, want):
            assert torch.equal(a, c)
        torch.cuda.synchronize()


def every_call():
    """Outputs of each operator on plain and on unusual arguments."""
    g = torch.Generator(device="cuda").manual_seed(4)
    r = lambda *shape: torch.randn(shape, device="cuda", generator=g)  # noqa: E731
    x, w, b, z = r(2, 9, 24), r(40, 24), r(40), r(2, 9, 40)
    out = []
    for cast in (lambda t: t, lambda t: t.to(torch.bfloat16), lambda t: torch.nn.Parameter(t), lambda t: t[..., ::1].flip(0).flip(0)):
        X, W, Z = cast(x), cast(w), cast(z)
        out += [*ops.linear(X, W, b, Z, activation="gelu", p=0.2, seed=1, offset=2, keep_pre=True), ops.linear(X, W), ops.linear(X[0, 0], W)]
        out += [ops.linear_input_grad(Z, W, pre=X, activation="silu", p=0.1, seed=3, offset=1, residual=X), ops.linear_input_grad(Z, W)]
        out += [*ops.linear_weight_grad(Z, X), *ops.linear_weight_grad(Z, X, torch.ones(40, 24, device="cuda"), torch.ones(40, device="cuda"), accumulate=True)]
        out += [ops.linear_weight_grad(Z, X, bias=False)[0], ops.dropout(X, 0.5, 1, 1, residual=X), ops.dropout_grad(X, 0.5, 1, 1), ops.dropout(X[0, 0], 0.5, 1, 1)]
        y, mean, rstd = ops.group_norm(X, 4, b[:24], b[:24], activation="relu")
        out += [y, mean, rstd, *ops.group_norm_grad(X, X, mean, rstd, 4, b[:24]), *ops.group_norm(X[0], 1)]
        out += ops.group_norm_grad(X, X, mean, rstd, 4, residual=X, dweight=torch.ones(24, device="cuda"), dbias=torch.ones(24, device="cuda"), accumulate=True)
    return out


def test_arguments_looked_at_in_python_give_the_same(monkeypatch):
    native = every_call()
    monkeypatch.setattr(ops, "_native", None)
    assert not ops._is_native()
    for a, b in zip(native, every_call()):
        assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b)


@pytest.mark.parametrize("native", [True, False])
def test_refusals(native, monkeypatch):
    if not native:
        monkeypatch.setattr(ops, "_native", None)
        assert not ops._is_native()
    x, w = torch.randn((4, 8), device="cuda"), torch.randn((6, 8), device="cuda")
    bad = [
        lambda: ops.linear(x.cpu(), w), lambda: ops.linear(x, w.cpu()), lambda: ops.linear(x, w.half()), lambda: ops.linear(x.half(), w.half()),
        lambda: ops.linear(x.double(), w.double()), lambda: ops.linear(x, w.t()), lambda: ops.linear(x, torch.randn((6, 9), device="cuda")),
        lambda: ops.linear(x, w, torch.zeros(7, device="cuda")), lambda: ops.linear(x, w, torch.zeros(6, dtype=torch.bfloat16, device="cuda")),
        lambda: ops.linear(x, w, residual=x), lambda: ops.linear(x, w, activation="tanh"), lambda: ops.linear(x, w, seed=-1),
        lambda: ops.linear(x, w, offset=1 << 64), lambda: ops.linear(torch.tensor(1.0, device="cuda"), w),
        lambda: ops.linear(torch.randn((4, 4, 16), device="cuda")[:, ::2, ::2], w), lambda: ops.linear_input_grad(x, w, pre=x, activation="relu"),
        lambda: ops.linear_weight_grad(x, torch.randn((5, 3), device="cuda")), lambda: ops.linear_weight_grad(x, x, accumulate=True),
        lambda: ops.linear_weight_grad(x, x, dweight=torch.zeros((8, 8), dtype=torch.bfloat16, device="cuda")),
        lambda: ops.dropout(x, 0.1, 1, 1, residual=w), lambda: ops.dropout(x[:, ::2], 0.1, 1, 1),
        lambda: ops.group_norm(x[0], 1), lambda: ops.group_norm(x, 1, torch.ones(7, device="cuda")),
        lambda: ops.group_norm(torch.randn((2, 8, 4), device="cuda").transpose(1, 2), 1), lambda: ops.group_norm_grad(w, x, x, x, 1),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was not refused")
    for call in (lambda: ops.linear(x, w, p=1.5), lambda: ops.linear(x, w, p=float("nan")), lambda: ops.linear(x.new_zeros(1, 8).expand(4, 8), w),
                 lambda: ops.group_norm(x, 3), lambda: ops.group_norm(x, 0), lambda: ops.group_norm(x, 1, eps=-1.0),
                 lambda: ops.linear_input_grad(torch.randn((4, 6), device="cuda"), w, activation="gelu"),
                 lambda: ops.dropout_grad(x, 0.1, 1, 1, activation="silu"), lambda: ops.dropout(x, -0.1, 1, 1)):
        with pytest.raises(qoda.QodaError) as e:
            call()
        assert e.value.code == qoda.EINVAL and len(ops.operator_error()) > 10
    torch.cuda.synchronize()
    assert torch.isfinite(ops.linear(x, w)).all()
