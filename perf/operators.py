"""The operators between two rounds of the optimiser, as cases that can be timed and whose outputs can be compared.

A node's dual vector is the gradient of its model's loss.  These are the operators of that model's blocks and their gradients:
the matrix product with bias, activation, dropout and residual in its epilogue; dropout whose mask comes from a counter-based
generator and is never stored; group normalisation with an activation, channels last (with one position and one group it is the
layer normalisation of the Transformer-shaped workloads).  Gradients of parameters are fp32, as the quantizer reads them.

``run`` computes a case either by the operators' plain form (elementary torch operations in 32 bits, one rounding at the end) or,
where ``own`` is true, by the library.  ``exact`` has the definitions in 64 bits, written apart from the plain form.

    linear          z = x W^T + b,  y = residual + drop(act(z));  z is kept for the gradient where ``pre`` says so
    input_grad      dx = residual + drop((dz W) * act'(pre))      (pre: the input of the activation that made x)
    weight_grad     dW = dz^T x,  db = the sum of dz's rows
    dropout         y = residual + drop(act(x))
    dropout_grad    dz = drop(dy * act'(pre))
    norm            h = (v - mean) * rstd * w + b,  y = act(h), mean and rstd per sample and group
    norm_grad       dx (+ residual), dw, db

drop: entry (r, c) of a matrix is kept where its lot is at least T = floor(p 65536 + 1/2), and then multiplied by
65536 / (65536 - T); otherwise the entry is 0, whatever it was.  Lots are 16-bit pieces of Philox4x32-10 with the counter
(c >> 3, r, offset low, offset high) and the key seed xor KEY: lot c & 7 is the low half of word c & 3, or its high half if
c & 4.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
KEY = 0x64726F706F757473
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = ("none", "relu", "leaky_relu", "gelu", "silu")
EPS = 1e-5
SLOPE = 0.2


# --------------------------------------------------------------------------------------------------- the cases
def _matrix(name, op, dtype, rows, cin, cout, act="none", p=0.0, residual=False, pre=False, pad=0):
    return dict(name=name, op=op, dtype=dtype, rows=rows, cin=cin, cout=cout, act=act, p=p, residual=residual, pre=pre, pad=pad)


def _entries(name, op, dtype, rows, cols, act="none", p=0.1, residual=False, pad=0):
    return dict(name=name, op=op, dtype=dtype, rows=rows, cols=cols, act=act, p=p, residual=residual, pad=pad)


def _norm(name, op, dtype, samples, positions, channels, groups, act="none", residual=False):
    return dict(name=name, op=op, dtype=dtype, samples=samples, positions=positions, channels=channels, groups=groups, act=act,
                residual=residual)


def listed():
    return [
        # one row through the wide matrix of the GPT-1.3B-shaped block, as when its samples are looked at between rounds: the
        # matrix is read once, latency counts
        _matrix("gpt_up_one_row", "linear", "bf16", 1, 2048, 8192, act="gelu"),
        # a small fp32 network of odd widths, one batch: launches and latency are all of it
        _matrix("small_block_f32", "linear", "f32", 37, 61, 61, act="relu", p=0.1, residual=True, pre=True),
        # Transformer-XL-sized feed-forward, 22 sequences of 150 tokens: rows of 410 entries end inside every tile and start
        # at 4-byte addresses
        _matrix("txl_up", "linear", "bf16", 3300, 410, 2100, act="relu", p=0.1, pre=True),
        # GPT-1.3B-shaped feed-forward, the way down, with the block's dropout and residual
        _matrix("gpt_down", "linear", "bf16", 16384, 8192, 2048, p=0.1, residual=True),
        # the gradient of the same product, through the dropout-free activation before it
        _matrix("gpt_down_input_grad", "input_grad", "bf16", 8192, 8192, 2048, act="gelu", p=0.0, pre=True),
        # the gradient of the fused query-key-value matrix, 8 sequences of 1024 tokens
        _matrix("gpt_qkv_weight_grad", "weight_grad", "bf16", 8192, 2048, 6144),
        # Transformer-XL-sized in fp32, the type that the optimiser's own parameters have
        _matrix("txl_up_weight_grad_f32", "weight_grad", "f32", 3300, 410, 2100),
        # dropout of the Transformer-XL-sized embedding
        _entries("txl_embedding_dropout", "dropout", "bf16", 3300, 410),
        # back through dropout and activation, the widest matrix of the GPT-1.3B-shaped model, 16 sequences of 2048 tokens
        _entries("gpt_wide_dropout_grad", "dropout_grad", "bf16", 32768, 8192, act="gelu"),
        # a critic's feature map, 64 images of 16 x 16 with 256 channels, fp32
        _norm("dcgan_norm", "norm", "f32", 64, 256, 256, 32, act="leaky_relu"),
        # the gradient at the larger map, 128 images of 32 x 32 with 128 channels
        _norm("dcgan_norm_grad", "norm_grad", "bf16", 128, 1024, 128, 32, act="silu"),
        # layer normalisation of the GPT-1.3B-shaped block, its gradient added to the residual's
        _norm("gpt_layer_norm_grad", "norm_grad", "bf16", 16384, 1, 2048, 1, residual=True),
    ]


def _spread(rng, lo, hi):
    """A whole number, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A width: odd sizes, and those that are multiples of 2, 8 and 64."""
    w = _spread(rng, lo, hi)
    m = rng.choice([1, 1, 2, 8, 64])
    return max(lo, w // m * m)


def draw(rng):
    op = rng.choice(["linear"] * 4 + ["input_grad"] * 3 + ["weight_grad"] * 3 + ["dropout", "dropout_grad"] * 2 + ["norm", "norm_grad"] * 3)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    p = rng.choice([0.0, 0.1, 0.1, 0.2, 0.5])
    if op in ("linear", "input_grad", "weight_grad"):
        cin, cout = _width(rng, 16, 8192), _width(rng, 16, 8192)
        most = min(16384, int((5e11 if dtype == "bf16" else 1e11) / (2.0 * cin * cout)))
        rows = rng.choice([1, 2, 5, 16, 33]) if rng.random() < 0.2 else _spread(rng, 16, max(17, most))
        pre = op != "weight_grad" and rng.random() < 0.5
        act = "none" if op == "weight_grad" or (op == "input_grad" and not pre) else rng.choice(ACTS)
        case = _matrix("", op, dtype, rows, cin, cout, act=act, p=0.0 if op == "weight_grad" else p,
                       residual=op != "weight_grad" and rng.random() < 0.5, pre=pre, pad=rng.choice([0, 0, 0, 1, 24]))
    elif op in ("dropout", "dropout_grad"):
        cols = _width(rng, 16, 16384)
        rows = _spread(rng, 1, max(2, min(65536, int(1.2e8 / cols))))
        case = _entries("", op, dtype, rows, cols, act=rng.choice(ACTS), p=rng.choice([0.1, 0.1, 0.2, 0.5]),
                        residual=op == "dropout" and rng.random() < 0.5, pad=rng.choice([0, 0, 0, 1, 24]))
    else:
        # the gradient of a kink at a value computed in the same pass is not to be compared between two roundings
        act = rng.choice(("none", "gelu", "silu") if op == "norm_grad" else ACTS)
        if rng.random() < 0.5:                          # layer normalisation
            channels, groups, positions = _width(rng, 16, 16384), 1, 1
            samples = _spread(rng, 1, max(2, min(65536, int(6e7 / channels))))
        else:                                           # feature maps
            groups = rng.choice([1, 2, 8, 16, 32])
            channels = groups * _spread(rng, 1, max(2, 1024 // groups))
            side = _spread(rng, 2, 64)
            positions = side * (side + rng.choice([0, 0, 1]))
            samples = _spread(rng, 1, max(2, min(256, int(3e7 / (channels * positions)))))
        case = _norm("", op, dtype, samples, positions, channels, groups, act=act, residual=op == "norm_grad" and rng.random() < 0.3)
    del case["name"]
    return case


# ------------------------------------------------------------------------------------------------------ inputs
def _heavy(shape, gen):
    """Student-t with 3 degrees of freedom, the distribution of the library's synthetic dual vectors."""
    chi = torch.zeros(shape, device=DEV)
    for _ in range(3):
        chi += torch.randn(shape, device=DEV, generator=gen).square_()
    return torch.randn(shape, device=DEV, generator=gen).mul_(chi.div_(3.0).rsqrt_())


def _rows(values, dtype, pad):
    """The values as a matrix of this type whose rows are ``pad`` entries further apart than they are long."""
    if not pad:
        return values.to(dtype)
    wide = torch.zeros((values.shape[0], values.shape[1] + pad), dtype=dtype, device=DEV)
    view = wide[:, : values.shape[1]]
    view.copy_(values)
    return view


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed) % (1 << 62))
    dt, op = TYPES[case["dtype"]], case["op"]
    normal = lambda *shape: torch.randn(shape, device=DEV, generator=gen)  # noqa: E731
    st = {"case": case, "seed": int(seed) * 2654435761 % (1 << 64), "offset": (7 << 32) + int(seed) % 1000}
    if op in ("linear", "input_grad", "weight_grad"):
        rows, cin, cout, pad = case["rows"], case["cin"], case["cout"], case["pad"]
        if op == "linear":
            st["x"] = _rows(normal(rows, cin), dt, pad)
            st["w"] = _rows(normal(cout, cin) / math.sqrt(cin), dt, pad)
            st["b"] = normal(cout) * 0.1
            st["residual"] = _rows(normal(rows, cout), dt, pad) if case["residual"] else None
        elif op == "input_grad":
            st["dz"] = _rows(_heavy((rows, cout), gen) * 1e-3, dt, pad)
            st["w"] = _rows(normal(cout, cin) / math.sqrt(cout), dt, pad)
            st["pre"] = _rows(normal(rows, cin), dt, pad) if case["pre"] else None
            st["residual"] = _rows(_heavy((rows, cin), gen) * 1e-3, dt, pad) if case["residual"] else None
        else:
            st["dz"] = _rows(_heavy((rows, cout), gen) * 1e-3, dt, pad)
            st["x"] = _rows(normal(rows, cin), dt, pad)
            # one flat fp32 vector that the quantizer reads, the two tensors at 256-byte boundaries of it
            st["dw"] = torch.zeros(cout * cin, device=DEV).view(cout, cin)
            st["db"] = torch.zeros(cout, device=DEV)
    elif op == "dropout":
        st["x"] = _rows(normal(case["rows"], case["cols"]), dt, case["pad"])
        st["residual"] = _rows(normal(case["rows"], case["cols"]), dt, case["pad"]) if case["residual"] else None
    elif op == "dropout_grad":
        st["dy"] = _rows(_heavy((case["rows"], case["cols"]), gen) * 1e-3, dt, case["pad"])
        st["pre"] = _rows(normal(case["rows"], case["cols"]), dt, case["pad"]) if case["act"] != "none" else None
    else:
        n, s, c, g = case["samples"], case["positions"], case["channels"], case["groups"]
        # channels of different spread and mean, as a trained layer leaves them
        st["x"] = (normal(n, s, c) * (0.5 + normal(c).abs()) + normal(c)).to(dt)
        st["w"], st["b"] = 1.0 + 0.2 * normal(c), 0.2 * normal(c)
        if op == "norm_grad":
            st["dy"] = (_heavy((n, s, c), gen) * 1e-3).to(dt)
            st["residual"] = (_heavy((n, s, c), gen) * 1e-3).to(dt) if case["residual"] else None
            # what the forward pass has kept
            var, mean = torch.var_mean(st["x"].double().view(n, s, g, c // g), dim=(1, 3), unbiased=False)
            st["mean"], st["rstd"] = mean.float(), (var + EPS).rsqrt().float()
    return st


# -------------------------------------------------------------------------------------------------- plain form
def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "leaky_relu":
        return torch.where(z > 0, z, SLOPE * z)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * (1.0 / math.sqrt(2.0))))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    """The activation's derivative; that from the left at a kink."""
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "leaky_relu":
        return torch.where(z > 0, 1.0, SLOPE).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * (1.0 / math.sqrt(2.0)))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def _threshold(p):
    return int(math.floor(p * 65536.0 + 0.5))


def _signed(v):
    """A 64-bit pattern as torch's signed whole number."""
    return v - (1 << 64) if v >= 1 << 63 else v


def _lots(rows, cols, seed, offset):
    """The 16-bit lots of a matrix: Philox4x32-10 in 64-bit products, whose low and high words are what is wanted."""
    mask, key = 0xFFFFFFFF, (seed ^ KEY)
    k0, k1 = key & mask, key >> 32
    blocks = (cols + 7) // 8
    c0 = torch.arange(blocks, dtype=torch.int64, device=DEV).expand(rows, blocks)
    c1 = torch.arange(rows, dtype=torch.int64, device=DEV)[:, None].expand(rows, blocks)
    c2, c3 = torch.full_like(c0, offset & mask), torch.full_like(c0, offset >> 32)
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & mask) ^ c1 ^ k0, p1 & mask, ((p0 >> 32) & mask) ^ c3 ^ k1, p0 & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    words = torch.stack((c0, c1, c2, c3), dim=-1)
    return torch.cat((words & 0xFFFF, words >> 16), dim=-1).view(rows, blocks * 8)[:, :cols]


def _drop(v, p, seed, offset):
    t = _threshold(p)
    if t == 0:
        return v
    kept = _lots(v.shape[0], v.shape[1], seed, offset) >= t
    return torch.where(kept, v * (65536.0 / (65536 - t) if t < 65536 else 0.0), 0.0)


def _plain(st):
    case, op, dt = st["case"], st["case"]["op"], TYPES[st["case"]["dtype"]]
    res = st.get("residual")
    if op == "linear":
        z = st["x"].float() @ st["w"].float().t() + st["b"]
        y = _drop(_act(z, case["act"]), case["p"], st["seed"], st["offset"])
        y = y if res is None else res.float() + y
        return {"y": y.to(dt), "pre": z.to(dt)} if case["pre"] else {"y": y.to(dt)}
    if op == "input_grad":
        dx = st["dz"].float() @ st["w"].float()
        dx = dx if st["pre"] is None else dx * _act_slope(st["pre"].float(), case["act"])
        dx = _drop(dx, case["p"], st["seed"], st["offset"])
        return {"dx": (dx if res is None else res.float() + dx).to(dt)}
    if op == "weight_grad":
        dz = st["dz"].float()
        return {"dw": dz.t() @ st["x"].float(), "db": dz.sum(0)}
    if op == "dropout":
        y = _drop(_act(st["x"].float(), case["act"]), case["p"], st["seed"], st["offset"])
        return {"y": (y if res is None else res.float() + y).to(dt)}
    if op == "dropout_grad":
        dz = st["dy"].float()
        dz = dz if st["pre"] is None else dz * _act_slope(st["pre"].float(), case["act"])
        return {"dz": _drop(dz, case["p"], st["seed"], st["offset"]).to(dt)}
    n, s, c, g = case["samples"], case["positions"], case["channels"], case["groups"]
    x = st["x"].float().view(n, s, g, c // g)
    w, b = st["w"].view(g, c // g), st["b"].view(g, c // g)
    if op == "norm":
        mean = x.mean(dim=(1, 3))
        d = x - mean[:, None, :, None]
        rstd = 1.0 / torch.sqrt((d * d).mean(dim=(1, 3)) + EPS)
        y = _act(d * rstd[:, None, :, None] * w + b, case["act"])
        return {"y": y.view(n, s, c).to(dt), "mean": mean, "rstd": rstd}
    rstd = st["rstd"][:, None, :, None]
    xhat = (x - st["mean"][:, None, :, None]) * rstd
    dh = st["dy"].float().view(n, s, g, c // g)
    dh = dh if case["act"] == "none" else dh * _act_slope(xhat * w + b, case["act"])
    dxhat = dh * w
    m1, m2 = dxhat.mean(dim=(1, 3), keepdim=True), (dxhat * xhat).mean(dim=(1, 3), keepdim=True)
    dx = ((dxhat - m1 - xhat * m2) * rstd).view(n, s, c)
    return {"dx": (dx if res is None else res.float() + dx).to(dt), "dw": (dh * xhat).sum(dim=(0, 1)).view(c), "db": dh.sum(dim=(0, 1)).view(c)}


# ----------------------------------------------------------------------------------------------------- a pass
def _library(st):
    from paper_2505_14371_amd import operators as ops

    case, op = st["case"], st["case"]["op"]
    drop = {"activation": case["act"], "p": case["p"], "seed": st["seed"], "offset": st["offset"]} if "p" in case else {}
    if op == "linear":
        out = ops.linear(st["x"], st["w"], st["b"], residual=st["residual"], keep_pre=case["pre"], **drop)
        return {"y": out[0], "pre": out[1]} if case["pre"] else {"y": out}
    if op == "input_grad":
        return {"dx": ops.linear_input_grad(st["dz"], st["w"], pre=st["pre"], residual=st["residual"], **drop)}
    if op == "weight_grad":
        dw, db = ops.linear_weight_grad(st["dz"], st["x"], dweight=st["dw"], dbias=st["db"])
        return {"dw": dw, "db": db}
    if op == "dropout":
        return {"y": ops.dropout(st["x"], residual=st["residual"], **drop)}
    if op == "dropout_grad":
        return {"dz": ops.dropout_grad(st["dy"], pre=st["pre"], **drop)}
    if op == "norm":
        y, mean, rstd = ops.group_norm(st["x"], case["groups"], st["w"], st["b"], eps=EPS, activation=case["act"])
        return {"y": y, "mean": mean, "rstd": rstd}
    dx, dw, db = ops.group_norm_grad(st["dy"], st["x"], st["mean"], st["rstd"], case["groups"], st["w"], st["b"],
                                     activation=case["act"], residual=st["residual"])
    return {"dx": dx, "dw": dw, "db": db}


def run(state):
    return _library(state) if own else _plain(state)


def work(case):
    e, op = 2 if case["dtype"] == "bf16" else 4, case["op"]
    if op in ("linear", "input_grad", "weight_grad"):
        rows, cin, cout = case["rows"], case["cin"], case["cout"]
        a, b, w = rows * cin, rows * cout, cin * cout
        flops = 2.0 * rows * cin * cout
        if op == "linear":
            return {"bytes": e * (a + w + b * (1 + case["residual"] + case["pre"])) + 4 * cout, "flops": flops}
        if op == "input_grad":
            return {"bytes": e * (b + w + a * (1 + case["residual"] + case["pre"])), "flops": flops}
        return {"bytes": e * (a + b) + 4 * (w + cout), "flops": flops}
    if op in ("dropout", "dropout_grad"):
        read = 1 + case["residual"] if op == "dropout" else 1 + (case["act"] != "none")
        n = case["rows"] * case["cols"]
        return {"bytes": e * n * (read + 1), "flops": 10.0 * n}
    n = case["samples"] * case["positions"] * case["channels"]
    if op == "norm":
        return {"bytes": e * 2 * n + 8 * case["channels"] + 8 * case["samples"] * case["groups"], "flops": 10.0 * n}
    return {"bytes": e * (3 + case["residual"]) * n + 16 * case["channels"] + 8 * case["samples"] * case["groups"], "flops": 20.0 * n}


# ----------------------------------------------------------------------------------------- the definitions, 64 bits
def _mul32(a, b):
    """(high, low) words of the product of two 32-bit numbers, from products of 16 bits."""
    al, ah, bl, bh = a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16
    mid = ah * bl + (al * bl >> 16)
    low = (mid & 0xFFFF) + al * bh
    return (ah * bh + (mid >> 16) + (low >> 16)), ((low & 0xFFFF) << 16) | (al * bl & 0xFFFF)


def _factor(case, st, rows, cols):
    """What dropout multiplies every entry of a matrix with, in 64 bits (0: dropped)."""
    t = int(np.floor(case["p"] * 65536 + 0.5))
    if t == 0:
        return torch.ones((), dtype=torch.float64, device=DEV)
    key = (st["seed"] ^ KEY)
    out = torch.empty((rows, cols), dtype=torch.float64, device=DEV)
    piece = max(1, (1 << 25) // cols)
    for r0 in range(0, rows, piece):
        r = torch.arange(r0, min(rows, r0 + piece), device=DEV)[:, None]
        c = torch.arange(0, cols, 8, device=DEV)[None, :]
        w = [(c + 0 * r) // 8, r + 0 * c, 0 * (r + c) + st["offset"] % 2**32, 0 * (r + c) + st["offset"] // 2**32]
        for i in range(10):
            ka, kb = (key % 2**32 + i * 0x9E3779B9) % 2**32, (key // 2**32 + i * 0xBB67AE85) % 2**32
            (h0, l0), (h1, l1) = _mul32(w[0], 0xD2511F53), _mul32(w[2], 0xCD9E8D57)
            w = [h1 ^ w[1] ^ ka, l1, h0 ^ w[3] ^ kb, l0]
        for lot in range(min(8, cols)):
            v = w[lot % 4] % 65536 if lot < 4 else w[lot % 4] // 65536
            at = out[r0: r0 + r.shape[0], lot::8]
            at.copy_(((v >= t).double() * (65536.0 / (65536 - t) if t < 65536 else 0.0))[:, : at.shape[1]])
    return out


def _exact_act(z, act):
    if act == "relu":
        return torch.maximum(z, torch.zeros_like(z))
    if act == "leaky_relu":
        return torch.maximum(z, SLOPE * z)
    if act == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _exact_slope(z, act):
    if act in ("relu", "leaky_relu"):
        low = torch.full_like(z, 0.0 if act == "relu" else SLOPE)
        return torch.where(z > 0, torch.ones_like(z), low)
    if act == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2.0)) + z / math.sqrt(2.0 * math.pi) * torch.exp(-z.square() / 2)
    if act == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    return torch.ones_like(z)


def exact(case, seed):
    st, op = prepare(case, seed), case["op"]
    wide = lambda k: st[k].double() if st.get(k) is not None else 0.0  # noqa: E731
    if op == "linear":
        z = torch.matmul(wide("x"), wide("w").t().contiguous()) + wide("b")
        y = wide("residual") + _exact_act(z, case["act"]) * _factor(case, st, *z.shape)
        return {"y": y, "pre": z} if case["pre"] else {"y": y}
    if op == "input_grad":
        dx = torch.matmul(wide("dz"), wide("w"))
        dx *= _factor(case, st, *dx.shape)
        return {"dx": (dx if st["pre"] is None else dx * _exact_slope(wide("pre"), case["act"])) + wide("residual")}
    if op == "weight_grad":
        return {"dw": torch.matmul(wide("dz").t().contiguous(), wide("x")), "db": wide("dz").sum(0)}
    if op == "dropout":
        y = _exact_act(wide("x"), case["act"])
        return {"y": y * _factor(case, st, *y.shape) + wide("residual")}
    if op == "dropout_grad":
        dz = wide("dy")
        dz = dz * _factor(case, st, *dz.shape)
        return {"dz": dz if st["pre"] is None else dz * _exact_slope(wide("pre"), case["act"])}
    n, s, c, g = case["samples"], case["positions"], case["channels"], case["groups"]
    x = wide("x").view(n, s, g, c // g).transpose(1, 2).reshape(n, g, -1)            # a row of values for each mean
    per = lambda v: v.view(g, 1, c // g).expand(g, s, c // g).reshape(g, -1)  # noqa: E731
    back = lambda v: v.view(n, g, s, c // g).transpose(1, 2).reshape(n, s, c)  # noqa: E731
    if op == "norm":
        var, mean = torch.var_mean(x, dim=-1, unbiased=False, keepdim=True)
        rstd = (var + EPS) ** -0.5
        y = _exact_act((x - mean) * rstd * per(wide("w")) + per(wide("b")), case["act"])
        return {"y": back(y), "mean": mean.view(n, g), "rstd": rstd.view(n, g)}
    mean, rstd = wide("mean")[..., None], wide("rstd")[..., None]
    xhat = (x - mean) * rstd
    dh = wide("dy").view(n, s, g, c // g).transpose(1, 2).reshape(n, g, -1)
    dh = dh * _exact_slope(xhat * per(wide("w")) + per(wide("b")), case["act"])
    u = dh * per(wide("w"))
    dx = rstd * (u - u.mean(-1, keepdim=True) - xhat * (u * xhat).mean(-1, keepdim=True))
    return {"dx": back(dx) + wide("residual"), "dw": back(dh * xhat).sum((0, 1)), "db": back(dh).sum((0, 1))}
