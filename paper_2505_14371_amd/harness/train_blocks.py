"""Residual blocks trained by K nodes whose gradients are quantized: every operator of the step is one of the library's.

    python -m paper_2505_14371_amd.harness.train_blocks [--width 512] [--hidden 2048] [--depth 4] [--nodes 4] [--rows 2048] [--rounds 60]

The task is synthetic: the rows of a fixed random two-layer map, to be matched.  The loss is a row's sum of squares, in the mean over the
rows and the nodes.  Prints the loss and the time of a round, and what part of it the model and the optimiser take.
"""
from __future__ import annotations

import argparse
import time

import torch

from ..blocks import ResidualBlocks
from ..solver import QODA


def batch(width: int, rows: int, nodes: int, seed: int, dtype):
    """Every node's inputs and targets: the same map for all, other rows for each."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda *shape: torch.randn(shape, device="cuda", generator=gen)  # noqa: E731
    a, b = draw(width, width) * width ** -0.5, draw(width, width) * width ** -0.5
    x = [draw(rows, width) for _ in range(nodes)]
    return [v.to(dtype) for v in x], [v + torch.tanh(v @ a) @ b for v in x]


def loss_of(y: torch.Tensor, target: torch.Tensor):
    """(a node's loss, its gradient by y in y's type)"""
    off, rows = y.float() - target, target.numel() // target.shape[-1]
    return off.square().sum() / rows, (off * (2.0 / rows)).to(y.dtype)


def train(width=512, hidden=2048, depth=4, nodes=4, rows=2048, rounds=60, points=16, p=0.1, dtype=torch.bfloat16, seed=0):
    """(losses of the rounds, seconds of a round, seconds of its model part): medians over the rounds behind the first three."""
    model = ResidualBlocks(width, hidden, depth, p=p, dtype=dtype, seed=seed)
    opt = QODA(model.params, num_nodes=nodes, points=points, seed=seed, fit_every=10)
    grads = [model.gradients() for _ in range(nodes)]
    x, target = batch(width, rows, nodes, seed, dtype)
    losses, whole, part = [], [], []
    for t in range(rounds):
        torch.cuda.synchronize()
        start = time.perf_counter()
        weights = model.weights()
        loss = torch.zeros((), device="cuda")
        for k in range(nodes):
            y, saved = model.forward(x[k], weights, draw=t * nodes + k)
            one, dy = loss_of(y, target[k])
            loss += one / nodes
            model.backward(dy, saved, weights, grads[k])
        torch.cuda.synchronize()
        part.append(time.perf_counter() - start)
        opt.step(grads)
        torch.cuda.synchronize()
        whole.append(time.perf_counter() - start)
        losses.append(float(loss))
    opt.close()
    mid = lambda v: sorted(v[3:] or v)[len(v[3:] or v) // 2]  # noqa: E731
    return losses, mid(whole), mid(part)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("width", 512), ("hidden", 2048), ("depth", 4), ("nodes", 4), ("rows", 2048), ("rounds", 60), ("points", 16)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--p", type=float, default=0.1)
    ap.add_argument("--f32", action="store_true", help="fp32 activations and products")
    a = vars(ap.parse_args())
    losses, whole, part = train(dtype=torch.float32 if a.pop("f32") else torch.bfloat16, **a)
    for t in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"round {t + 1}: loss {losses[t]:.5f}")
    print(f"last loss {losses[-1]:.5f}; {whole * 1e3:.3f} ms a round, {part * 1e3:.3f} of it forward and backward of the {a['nodes']} nodes")


if __name__ == "__main__":
    main()
