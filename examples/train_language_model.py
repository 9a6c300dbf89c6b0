"""n workers train a small language model over a lossy network, on one GPU.

Each worker holds a replica of the model in a row of the flat ``[n][pitch]`` array of ``RPS`` and sees its own text.  A step is

  1. the worker's own gradient, of all workers at once, by the training operators (``paper_1810_07766_b200.ops``): the words' rows of a table;
     blocks of linear attention with a decay for each head (``--heads``) and of two linear layers whose inputs are kept in 8 bits, the norms,
     gate and residual sum between the blocks in one kernel; the cross entropy over the vocabulary without the logits and, with
     ``--teacher``, the divergence from a teacher's largest logits as well;
  2. local SGD and the averaging over messages of which a fraction p is lost, by ``RPS.step``: with the targets set to b = x - g and no
     added noise its update x - gamma (x - b) is x - gamma g.

The text is synthetic: a fixed random successor for each word, followed with probability 0.9 (so the loss can fall from log V to
about 0.1 log V + 0.33).  The teacher knows the text's own probabilities.  At the end the first worker's model goes on with a few texts, each
word by one recurrent step of the attention.

    python examples/train_language_model.py --steps 200 --workers 4 --drop 0.1 --heads 2 --teacher 8
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


def decays(workers, heads):
    """From heads that forget within a few words to heads that remember hundreds; the same for all workers."""
    return torch.log1p(-torch.exp2(-2.0 - 6.0 * torch.arange(heads, device="cuda") / max(heads, 1))).repeat(workers, 1)


def attend(y, weights, heads, sequences, state=None):
    """One attention's output for y [n, tokens, width], the sequences one after another; with `state` for one new word of each sequence."""
    n, tokens, width = y.shape
    joint = ops.linear_8bit(y, weights["qkv"]).view(n, sequences, tokens // sequences, heads, -1)
    q, k, v = joint.chunk(3, -1)
    if state is None:
        out, state = ops.linear_attention(q, k, v, decays(n, heads))
    else:
        out = ops.linear_attention_step(q[:, :, 0], k[:, :, 0], v[:, :, 0], decays(n, heads), state)
    return ops.linear_8bit(out.reshape(n, tokens, width), weights["out"]), state


def features(p, tokens, blocks, keep, heads, sequences, states=None):
    """What the head reads, [n, tokens, width], and the attentions' states after the last word."""
    after = []

    def rejoin(x, f, name):
        return ops.gated_residual_norm(x, f, p[f"{name}.gate"], p[f"{name}.post"], p[f"{name}.pre"], scale=1.0 / math.sqrt(blocks), keep=keep)

    x = y = ops.embedding(tokens, p["embedding"])
    for i in range(blocks):
        if heads:
            f, state = attend(y, {name: p[f"{i}.{name}"] for name in ("qkv", "out")}, heads, sequences, states[i] if states else None)
            after.append(state)
            x, y = rejoin(x, f, f"{i}.mix")
        hidden = torch.relu(ops.linear_8bit(y, p[f"{i}.up"]))
        x, y = rejoin(x, ops.linear_8bit(hidden, p[f"{i}.down"]), i)
    return y, after


def model(p, tokens, targets, blocks, keep, heads=0, sequences=1, teacher=None):
    """Mean loss of each worker's text: the cross entropy, and half of each where there is a teacher: (ids, logits) of its largest."""
    y, _ = features(p, tokens, blocks, keep, heads, sequences)
    loss = ops.linear_cross_entropy(y, p["head"], targets)
    return loss if teacher is None else 0.5 * (loss + ops.linear_distillation(y, p["head"], *teacher))


def largest_logits(words, successor, vocab, top, generator):
    """The text's own probabilities as a teacher's: of the successor, and of some of the others, which are all alike."""
    ids = torch.randint(0, vocab, (*words.shape, top), generator=generator, device="cuda")
    first = successor[words][..., None]
    ids = torch.cat([first, torch.where(ids[..., 1:] == first, -100, ids[..., 1:])], -1)
    logits = torch.full(ids.shape, math.log(0.1 / vocab), device="cuda")
    logits[..., 0] = math.log(0.9)
    return ids, logits


@torch.no_grad()
def continue_texts(p, texts, words, blocks, heads):
    """The first worker's model goes on with the texts [sequences, tokens] by its most probable words, one at a time."""
    one = {name: leaf[:1] for name, leaf in p.items()}
    sequences = texts.shape[0]
    y, states = features(one, texts.reshape(1, -1), blocks, "values", heads, sequences)
    last = y.view(sequences, -1, y.shape[-1])[:, -1]
    out = []
    for _ in range(words):
        word = (last.float() @ one["head"][0].float().T).argmax(-1)
        out.append(word)
        y, _ = features(one, word[None], blocks, "values", heads, sequences, states)  # the states go on in place
        last = y[0]
    return torch.stack(out, 1)


def train(steps=100, workers=4, drop=0.1, gamma=0.5, vocab=1000, width=128, blocks=2, tokens=256, dtype="f32", keep="int8", seed=0, report=None, heads=0,
          sequences=1, teacher=0, further_words=0):
    """Runs the training; returns the workers' mean loss before each step (and, with `further_words`, texts that the first worker's model went on with)."""
    build.build()
    shapes = {"embedding": (vocab, width), "head": (vocab, width)}

    def norm(name):
        return {f"{name}.gate": (1, width), f"{name}.post": (width,), f"{name}.pre": (width,)}

    for i in range(blocks):
        shapes.update({f"{i}.up": (4 * width, width), f"{i}.down": (width, 4 * width), **norm(i)})
        if heads:
            shapes.update({f"{i}.qkv": (3 * width, width), f"{i}.out": (width, width), **norm(f"{i}.mix")})
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
        known = largest_logits(words, successor, vocab, teacher, g) if teacher else None
        loss = model(p, words, targets, blocks, keep, heads, sequences, known)
        loss.sum().backward()
        replicas.step(p)
        losses.append(loss.detach().mean())
        if report and t % report == 0:
            print(f"step {t}: loss {float(losses[-1]):.3f}", flush=True)
    ops.check()
    losses = torch.stack(losses).cpu()
    further = None
    if further_words:
        texts = torch.randint(0, vocab, (4, 8), generator=g, device="cuda")
        further = continue_texts(replicas.parameters(), texts, further_words, blocks, heads).cpu()
        ops.check()
    replicas.rps.close()
    return (losses, further) if further_words else losses


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
    ap.add_argument("--heads", type=int, default=2, help="heads of linear attention in each block; 0: none")
    ap.add_argument("--sequences", type=int, default=4, help="texts that a worker's tokens are")
    ap.add_argument("--teacher", type=int, default=0, help="largest logits of the teacher for each token; 0: none")
    ap.add_argument("--further-words", type=int, default=8, help="words that the trained model goes on with")
    a = ap.parse_args()
    out = train(**vars(a), report=20)
    if a.further_words:
        out, further = out
        print("texts go on with", further.tolist())
    print(f"loss {float(out[:10].mean()):.3f} in the first ten steps, {float(out[-10:].mean()):.3f} in the last ten")
