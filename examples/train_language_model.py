"""n workers train a small language model over a lossy network, on one GPU.

Each worker holds a replica of the model in a row of the flat ``[n][pitch]`` array of ``RPS`` and sees its own text.  A step is

  1. the worker's own gradient, of all workers at once, by the training operators (``paper_1810_07766_b200.ops``): blocks of two linear
     layers whose inputs are kept in 8 bits, the norms, gate and residual sum between the blocks in one kernel, and the
     cross entropy over the vocabulary without the logits;
  2. local SGD and the averaging over messages of which a fraction p is lost, by ``RPS.step``: with the targets set to b = x - g and no
     added noise its update x - gamma (x - b) is x - gamma g.

The text is synthetic: a fixed random successor for each word, followed with probability 0.9 (so the loss can fall from log V to
about 0.1 log V + 0.33).

    python examples/train_language_model.py --steps 200 --workers 4 --drop 0.1
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1810_07766_b200 import binding, build, ops  # noqa: E402


class Replicas:
    """The model's parameters as views into the workers' rows; every one starts at a multiple of 64 columns."""

    def __init__(self, shapes, workers, dtype, drop, gamma, seed):
        self.at, d = {}, 0
        for name, shape in shapes.items():
            self.at[name] = (d, shape)
            d += -(-math.prod(shape) // 64) * 64
        # the targets are written by kernels of this program right before the step: their copies wait for it (early_targets=1)
        self.rps = binding.RPS(workers, d, drop, gamma, seed, dtype=dtype, early_targets=1)
        self.workers = workers

    def view(self, flat, name):
        at, shape = self.at[name]
        return flat[:, at:at + math.prod(shape)].view(self.workers, *shape)

    def parameters(self):
        """Leaves that share the replicas' memory."""
        return {name: self.view(self.rps.x_dev, name).detach().requires_grad_() for name in self.at}

    def step(self, parameters):
        self.rps.b_dev.copy_(self.rps.x_dev)
        for name, leaf in parameters.items():
            self.view(self.rps.b_dev, name).sub_(leaf.grad)
        self.rps.step()


def model(p, tokens, targets, blocks, keep):
    """Mean loss of each worker's text."""
    n = tokens.shape[0]
    x = p["embedding"][torch.arange(n, device=tokens.device)[:, None], tokens]
    y = x
    for i in range(blocks):
        hidden = torch.relu(ops.linear_8bit(y, p[f"{i}.up"]))
        f = ops.linear_8bit(hidden, p[f"{i}.down"])
        x, y = ops.gated_residual_norm(x, f, p[f"{i}.gate"], p[f"{i}.post"], p[f"{i}.pre"], scale=1.0 / math.sqrt(blocks), keep=keep)
    return ops.linear_cross_entropy(y, p["head"], targets)


def train(steps=100, workers=4, drop=0.1, gamma=0.5, vocab=1000, width=128, blocks=2, tokens=256, dtype="f32", keep="int8", seed=0, report=None):
    """Runs the training; returns the workers' mean loss before each step."""
    build.build()
    shapes = {"embedding": (vocab, width), "head": (vocab, width)}
    for i in range(blocks):
        shapes.update({f"{i}.up": (4 * width, width), f"{i}.down": (width, 4 * width), f"{i}.gate": (1, width), f"{i}.post": (width,),
                       f"{i}.pre": (width,)})
    replicas = Replicas(shapes, workers, dtype, drop, gamma, seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    with torch.no_grad():
        for name, (_, shape) in replicas.at.items():  # all workers start from the same model
            one = torch.ones(shape, device="cuda") if shape[-2:-1] in ((), (1,)) else torch.randn(shape, generator=g, device="cuda") / math.sqrt(shape[-1])
            replicas.view(replicas.rps.x_dev, name).copy_(one.expand(workers, *shape))
    successor = torch.randperm(vocab, generator=g, device="cuda")
    losses = []
    for t in range(steps):
        text = torch.randint(0, vocab, (workers, tokens + 1), generator=g, device="cuda")
        follow = torch.rand(workers, tokens, generator=g, device="cuda") < 0.9
        words, targets = text[:, :-1], torch.where(follow, successor[text[:, :-1]], text[:, 1:])
        p = replicas.parameters()
        loss = model(p, words, targets, blocks, keep)
        loss.sum().backward()
        replicas.step(p)
        losses.append(loss.detach().mean())
        if report and t % report == 0:
            print(f"step {t}: loss {float(losses[-1]):.3f}", flush=True)
    ops.check()
    losses = torch.stack(losses).cpu()
    replicas.rps.close()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--drop", type=float, default=0.1)
    ap.add_argument("--gamma", type=float, default=0.5)
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--width", type=int, default=128)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--tokens", type=int, default=256)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    ap.add_argument("--keep", choices=("values", "int8"), default="int8")
    a = ap.parse_args()
    out = train(**vars(a), report=20)
    print(f"loss {float(out[:10].mean()):.3f} in the first ten steps, {float(out[-10:].mean()):.3f} in the last ten")
