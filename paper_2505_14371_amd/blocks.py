"""Residual feed-forward blocks on the library's operators: a model whose K nodes' dual vectors the optimiser quantizes.

    model = ResidualBlocks(width=512, hidden=2048, depth=4, p=0.1)
    opt = QODA(model.params, num_nodes=K, points=8, fit_every=10)       # the parameters are the query point
    nodes = [model.gradients() for _ in range(K)]                       # fp32 tensors inside one flat vector each
    for t in range(T):
        weights = model.weights()                                       # cast once a round, for all nodes
        for k in range(K):
            y, saved = model.forward(x[k], weights, draw=t * K + k)
            model.backward(dloss(y), saved, weights, nodes[k])          # weight gradients straight into node k's vector
        opt.step(nodes)

A block is  h + drop(W2 drop(act(W1 n + b1)) + b2)  with n the group normalisation of h (one group: layer normalisation).  Every
operator of it and of its gradient is one of ``operators``; activations, masks' factors, residuals and biases are in the products'
epilogues.

With four_bit=True the products are those of ``matrices``: weights and activations are rounded to four bits to nearest, gradients stochastically, so that
their mean over the draws is that of the products' own gradients.  ``orthogonalize`` replaces the gradients of a node's matrices by their orthogonalised
forms before the optimiser quantizes them.
"""
from __future__ import annotations

from typing import List, Sequence, Tuple

import torch

from . import matrices as mats
from . import operators as ops
from . import workloads

PER_BLOCK = 6       # tensors: norm's weight and bias, W1, b1, W2, b2


class ResidualBlocks:
    def __init__(self, width: int, hidden: int, depth: int, *, groups: int = 1, activation: str = "gelu", p: float = 0.1, dtype=torch.bfloat16,
                 seed: int = 0, device="cuda", four_bit: bool = False):
        """dtype: of activations and of the products' operands (the parameters themselves are fp32); seed: of the initial
        weights, of dropout and of stochastic rounding; four_bit: the products' operands are rounded to four bits."""
        if dtype not in ops.DTYPES:
            raise ValueError(f"ResidualBlocks: {dtype} is neither float32 nor bfloat16")
        if width % groups != 0:
            raise ValueError(f"ResidualBlocks: {groups} groups do not divide a width of {width}")
        self.width, self.hidden, self.depth, self.groups = width, hidden, depth, groups
        self.activation, self.p, self.dtype, self.seed, self.four_bit = activation, p, dtype, seed, four_bit
        gen = torch.Generator(device=device).manual_seed(seed)
        self.params: List[torch.Tensor] = []
        for _ in range(depth):
            self.params += [torch.ones(width, device=device), torch.zeros(width, device=device),
                            torch.randn((hidden, width), device=device, generator=gen) * width ** -0.5, torch.zeros(hidden, device=device),
                            torch.randn((width, hidden), device=device, generator=gen) * (2 * depth * hidden) ** -0.5, torch.zeros(width, device=device)]

    def gradients(self) -> List[torch.Tensor]:
        """One node's gradient tensors, shaped like the parameters, inside one flat fp32 vector (at 256-byte boundaries)."""
        off, n = workloads.padded_offsets([q.numel() for q in self.params])
        flat = torch.zeros(n, dtype=torch.float32, device=self.params[0].device)
        return [flat[int(o): int(o) + q.numel()].view(q.shape) for o, q in zip(off, self.params)]

    def _matrices(self, tensors: Sequence[torch.Tensor]) -> List[torch.Tensor]:
        return [q for i in range(self.depth) for q in (tensors[PER_BLOCK * i + 2], tensors[PER_BLOCK * i + 4])]

    def weights(self) -> list:
        """The matrices in the form that the products take: of the blocks' type, or in four bits with their transposes."""
        if self.four_bit:
            return [(mats.microscale(q), mats.microscale(q, transposed=True)) for q in self._matrices(self.params)]
        return [q.to(self.dtype) for q in self._matrices(self.params)]

    def orthogonalize(self, grads: Sequence[torch.Tensor], **polynomial) -> None:
        """The gradients of one node's matrices replaced by their orthogonalised forms, in place; polynomial: steps, coefficients and eps of
        matrices.orthogonalize.  The blocks' matrices of one kind are taken together where they lie evenly spaced, as in gradients()."""
        for kind in (0, 1):
            g = self._matrices(grads)[kind::2]
            if not g:
                return
            apart = [b.storage_offset() - a.storage_offset() for a, b in zip(g, g[1:])]
            if len({q.untyped_storage().data_ptr() for q in g}) == 1 and len(set(apart)) == 1 and apart[0] >= g[0].numel() and all(q.is_contiguous() for q in g):
                g = [torch.as_strided(g[0], (len(g), *g[0].shape), (apart[0], g[0].shape[1], 1))]
            for q in g:
                mats.orthogonalize(q, out=q, **polynomial)

    def _drop(self, draw: int, block: int, site: int) -> dict:
        return {"p": self.p, "seed": self.seed, "offset": (draw * self.depth + block) * 2 + site}

    def _round(self, d: torch.Tensor, transposed: bool, draw: int, block: int, site: int):
        """A gradient in four bits, its two roundings from draws of their own."""
        return mats.microscale(d, transposed=transposed, rounding="stochastic", seed=self.seed, offset=2 * self._drop(draw, block, site)["offset"] + transposed)

    def _weight_grad(self, d, x, dweight, dbias, accumulate: bool, draw: int, block: int, site: int) -> None:
        if self.four_bit:
            mats.mx_linear_weight_grad(self._round(d, True, draw, block, site), mats.microscale(x, transposed=True), dweight, dbias, accumulate=accumulate)
        else:
            ops.linear_weight_grad(d, x, dweight, dbias, accumulate=accumulate)

    def _input_grad(self, d, weight, draw: int, block: int, site: int, **through) -> torch.Tensor:
        if self.four_bit:
            return mats.mx_linear_input_grad(self._round(d, False, draw, block, site), weight[1], dtype=self.dtype, **through)
        return ops.linear_input_grad(d, weight, **through)

    def forward(self, x: torch.Tensor, weights: Sequence, draw: int) -> Tuple[torch.Tensor, list]:
        """The blocks' output for rows x [..., width], and what backward() needs.  draw: numbers the call; another one drops others."""
        saved = [draw]
        linear, w = (mats.mx_linear, [q for q, _ in weights]) if self.four_bit else (ops.linear, weights)
        h = x.reshape(-1, x.shape[-1])       # rows: the norm would take dimensions in between as positions of one sample
        for i in range(self.depth):
            gamma, beta, _, b1, _, b2 = self.params[PER_BLOCK * i: PER_BLOCK * (i + 1)]
            n, mean, rstd = ops.group_norm(h, self.groups, gamma, beta)
            a, z = linear(n, w[2 * i], b1, activation=self.activation, keep_pre=True, **self._drop(draw, i, 0))
            saved.append((h, n, mean, rstd, z, a))
            h = linear(a, w[2 * i + 1], b2, residual=h, **self._drop(draw, i, 1))
        return h.view(x.shape), saved

    def backward(self, dy: torch.Tensor, saved: list, weights: Sequence, grads: Sequence[torch.Tensor], accumulate: bool = False) -> torch.Tensor:
        """The gradient of x, and those of the parameters into (accumulate: added to) ``grads``."""
        draw, dh = saved[0], dy.reshape(-1, dy.shape[-1])
        for i in reversed(range(self.depth)):
            gamma, beta = self.params[PER_BLOCK * i: PER_BLOCK * i + 2]
            g_gamma, g_beta, g_w1, g_b1, g_w2, g_b2 = grads[PER_BLOCK * i: PER_BLOCK * (i + 1)]
            h, n, mean, rstd, z, a = saved[1 + i]
            d2 = ops.dropout_grad(dh, **self._drop(draw, i, 1))
            self._weight_grad(d2, a, g_w2, g_b2, accumulate, draw, i, 1)
            d1 = self._input_grad(d2, weights[2 * i + 1], draw, i, 1, pre=z, activation=self.activation, **self._drop(draw, i, 0))
            self._weight_grad(d1, n, g_w1, g_b1, accumulate, draw, i, 0)
            dn = self._input_grad(d1, weights[2 * i], draw, i, 0)
            dh, _, _ = ops.group_norm_grad(dn, h, mean, rstd, self.groups, gamma, beta, residual=dh, dweight=g_gamma, dbias=g_beta, accumulate=accumulate)
        return dh.view(dy.shape)
