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
"""
from __future__ import annotations

from typing import List, Sequence, Tuple

import torch

from . import operators as ops
from . import workloads

PER_BLOCK = 6       # tensors: norm's weight and bias, W1, b1, W2, b2


class ResidualBlocks:
    def __init__(self, width: int, hidden: int, depth: int, *, groups: int = 1, activation: str = "gelu", p: float = 0.1, dtype=torch.bfloat16,
                 seed: int = 0, device="cuda"):
        """dtype: of activations and of the products' operands (the parameters themselves are fp32); seed: of the initial
        weights and of dropout."""
        if dtype not in ops.DTYPES:
            raise ValueError(f"ResidualBlocks: {dtype} is neither float32 nor bfloat16")
        if width % groups != 0:
            raise ValueError(f"ResidualBlocks: {groups} groups do not divide a width of {width}")
        self.width, self.hidden, self.depth, self.groups = width, hidden, depth, groups
        self.activation, self.p, self.dtype, self.seed = activation, p, dtype, seed
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

    def weights(self) -> List[torch.Tensor]:
        """The matrices in the type that the products take."""
        return [q.to(self.dtype) for i in range(self.depth) for q in (self.params[PER_BLOCK * i + 2], self.params[PER_BLOCK * i + 4])]

    def _drop(self, draw: int, block: int, site: int) -> dict:
        return {"p": self.p, "seed": self.seed, "offset": (draw * self.depth + block) * 2 + site}

    def forward(self, x: torch.Tensor, weights: Sequence[torch.Tensor], draw: int) -> Tuple[torch.Tensor, list]:
        """The blocks' output for rows x [..., width], and what backward() needs.  draw: numbers the call; another one drops others."""
        saved = [draw]
        h = x.reshape(-1, x.shape[-1])       # rows: the norm would take dimensions in between as positions of one sample
        for i in range(self.depth):
            gamma, beta, _, b1, _, b2 = self.params[PER_BLOCK * i: PER_BLOCK * (i + 1)]
            n, mean, rstd = ops.group_norm(h, self.groups, gamma, beta)
            a, z = ops.linear(n, weights[2 * i], b1, activation=self.activation, keep_pre=True, **self._drop(draw, i, 0))
            saved.append((h, n, mean, rstd, z, a))
            h = ops.linear(a, weights[2 * i + 1], b2, residual=h, **self._drop(draw, i, 1))
        return h.view(x.shape), saved

    def backward(self, dy: torch.Tensor, saved: list, weights: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], accumulate: bool = False) -> torch.Tensor:
        """The gradient of x, and those of the parameters into (accumulate: added to) ``grads``."""
        draw, dh = saved[0], dy.reshape(-1, dy.shape[-1])
        for i in reversed(range(self.depth)):
            gamma, beta = self.params[PER_BLOCK * i: PER_BLOCK * i + 2]
            g_gamma, g_beta, g_w1, g_b1, g_w2, g_b2 = grads[PER_BLOCK * i: PER_BLOCK * (i + 1)]
            h, n, mean, rstd, z, a = saved[1 + i]
            d2 = ops.dropout_grad(dh, **self._drop(draw, i, 1))
            ops.linear_weight_grad(d2, a, g_w2, g_b2, accumulate=accumulate)
            d1 = ops.linear_input_grad(d2, weights[2 * i + 1], pre=z, activation=self.activation, **self._drop(draw, i, 0))
            ops.linear_weight_grad(d1, n, g_w1, g_b1, accumulate=accumulate)
            dn = ops.linear_input_grad(d1, weights[2 * i])
            dh, _, _ = ops.group_norm_grad(dn, h, mean, rstd, self.groups, gamma, beta, residual=dh, dweight=g_gamma, dbias=g_beta, accumulate=accumulate)
        return dh.view(dy.shape)
