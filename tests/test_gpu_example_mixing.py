"""The language-model example with attention, a teacher and texts that go on: it runs, its gradients are those of the same model in plain operations."""
import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    import train_language_model

    train_language_model.build.build()
    return train_language_model


@pytest.mark.parametrize("dtype,drop,heads,teacher", [("f32", 0.0, 2, 4), ("bf16", 0.1, 4, 0), ("bf16", 0.1, 2, 8)])
def test_it_runs(example, dtype, drop, heads, teacher):
    losses, further = example.train(steps=10, workers=3, drop=drop, vocab=150, width=64, blocks=2, tokens=96, dtype=dtype, heads=heads, sequences=3, teacher=teacher,
                                    further_words=5)
    assert len(losses) == 10 and torch.isfinite(losses).all()
    assert further.shape == (4, 5) and (further >= 0).all() and (further < 150).all()


def plain(p, tokens, targets, blocks, heads, sequences, teacher, decay):
    """The example's model of one worker in elementary operations."""
    def norm(z):
        return z / torch.sqrt((z * z).mean(-1, keepdim=True) + 1e-6)

    def rejoin(x, f, name):
        x = x + (1.0 / math.sqrt(blocks)) * p[f"{name}.gate"] * norm(f) * p[f"{name}.post"]
        return x, norm(x) * p[f"{name}.pre"]

    x = y = p["embedding"][tokens]
    for i in range(blocks):
        q, k, v = (y @ p[f"{i}.qkv"].T).view(sequences, -1, heads, 3 * y.shape[-1] // heads).chunk(3, -1)
        T = q.shape[1]
        apart = torch.arange(T, device="cuda")[:, None] - torch.arange(T, device="cuda")
        weight = torch.where(apart >= 0, torch.exp(decay[:, None, None].double() * apart.clamp(min=0)), 0.0)
        scores = torch.einsum("sihd,sjhd->shij", q, k) * weight / math.sqrt(q.shape[-1])
        f = torch.einsum("shij,sjhd->sihd", scores, v).reshape(len(tokens), -1) @ p[f"{i}.out"].T
        x, y = rejoin(x, f, f"{i}.mix")
        f = torch.relu(y @ p[f"{i}.up"].T) @ p[f"{i}.down"].T
        x, y = rejoin(x, f, str(i))
    z = torch.log_softmax(y @ p["head"].T, -1)
    loss = -z.gather(1, targets[:, None]).mean()
    ids, logits = teacher
    q = torch.softmax(logits.double().masked_fill(ids < 0, -math.inf), -1)
    near = (torch.special.xlogy(q, q) - q * z.gather(1, ids.clamp(min=0))).sum(-1).mean()
    return 0.5 * (loss + near)


def test_gradients_of_the_whole_model(example):
    """fp32 through four norms, three products and a softmax each way: errors of a few 2^-22 of the terms, kept below 2^-12 of a gradient's norm
    with "values"; kept in 8 bits, a half step of 1/254 of the largest of 128 (about 2^-7 of a value) in each weight gradient's input."""
    n, vocab, width, blocks, heads, sequences, tokens = 2, 90, 32, 2, 2, 3, 60
    g = torch.Generator(device="cuda").manual_seed(0)
    shapes = {"embedding": (vocab, width), "head": (vocab, width)}
    for i in range(blocks):
        shapes.update({f"{i}.up": (4 * width, width), f"{i}.down": (width, 4 * width), f"{i}.qkv": (3 * width, width), f"{i}.out": (width, width)})
        for name in (f"{i}", f"{i}.mix"):
            shapes.update({f"{name}.gate": (1, width), f"{name}.post": (width,), f"{name}.pre": (width,)})
    p = {name: (torch.randn(n, *shape, generator=g, device="cuda") / math.sqrt(shape[-1]) + (1.0 if len(shape) == 1 else 0.0)).requires_grad_() for name, shape in shapes.items()}
    text, targets = (torch.randint(0, vocab, (n, tokens), generator=g, device="cuda") for _ in range(2))
    successor = torch.randperm(vocab, generator=g, device="cuda")
    teacher = example.largest_logits(text, successor, vocab, 5, g)
    loss = example.model(p, text, targets, blocks, "values", heads, sequences, teacher)
    loss.sum().backward()
    for w in range(n):
        q = {name: leaf.detach()[w].double().requires_grad_() for name, leaf in p.items()}
        want = plain(q, text[w], targets[w], blocks, heads, sequences, (teacher[0][w], teacher[1][w]), example.decays(n, heads)[w])
        want.backward()
        assert abs(float(loss.detach()[w]) - float(want.detach())) <= 1e-5 * float(want.detach())
        for name, leaf in p.items():
            # the weight gradients of linear_8bit come out of inputs in 8 bits
            near = 2.0 ** -5 if name.split(".")[-1] in ("up", "down", "qkv", "out") else 2.0 ** -12
            assert (leaf.grad[w] - q[name].grad).norm() <= near * q[name].grad.norm(), name


def test_a_captured_training_pass(example):
    """Words, attention over texts of several lengths, the loss and a teacher, forward and backward in one CUDA graph that is replayed with other
    words in place, beside the same calls made one by one: the same bits."""
    ops = example.ops
    n, vocab, width, heads, sequences, tokens = 2, 300, 32, 2, 3, 140
    g = torch.Generator(device="cuda").manual_seed(2)
    table = torch.randn(n, vocab, width, generator=g, device="cuda").bfloat16()
    decay = example.decays(n, heads)
    lengths = torch.tensor([[140, 1, 77], [0, 139, 128]], device="cuda")
    words, targets = (torch.randint(0, vocab, (n, sequences * tokens), generator=g, device="cuda") for _ in range(2))
    ids = torch.randint(0, vocab, (n, sequences * tokens, 6), generator=g, device="cuda")
    kept = torch.randn(n, sequences * tokens, 6, generator=g, device="cuda")

    def gradients():
        leaf = table.detach().requires_grad_()
        x = ops.embedding(words, leaf).view(n, sequences, tokens, heads, width // heads)
        out, _ = ops.linear_attention(x, x, x, decay, lengths=lengths)
        y = out.reshape(n, sequences * tokens, width)
        loss = ops.linear_cross_entropy(y, leaf, targets) + ops.linear_distillation(y, leaf, ids, kept, temperature=2.0)
        return loss.detach(), torch.autograd.grad(loss.sum(), leaf)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        gradients()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, grad = gradients()
    for _ in range(3):
        words.copy_(torch.randint(0, vocab, words.shape, generator=g, device="cuda"))
        lengths.copy_(lengths.flip(0))
        graph.replay()
        want_loss, want_grad = gradients()
        assert torch.equal(loss, want_loss) and torch.equal(grad, want_grad) and torch.isfinite(grad).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_two_streams_at_once(example, dtype):
    """Two users of the operators on streams of their own, with nothing between them: each gets the bits that it gets alone."""
    ops = example.ops
    kind = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]

    def user(seed, n, vocab, width, heads, sequences, tokens, top):
        g = torch.Generator(device="cuda").manual_seed(seed)
        table = torch.randn(n, vocab, width, generator=g, device="cuda").to(kind)
        words = torch.randint(0, vocab, (n, sequences * tokens), generator=g, device="cuda")
        ids = torch.randint(0, vocab, (n, sequences * tokens, top), generator=g, device="cuda")
        kept = torch.randn(n, sequences * tokens, top, generator=g, device="cuda")
        dloss = torch.ones(n, device="cuda")
        decay = example.decays(n, heads)

        def call():
            x = ops.embedding_forward(words, table).view(n, sequences, tokens, heads, -1)
            out, state = ops.linear_attention_forward(x, x, x, decay)
            y = out.view(n, sequences * tokens, width)
            loss, lse = ops.linear_distillation_forward(y, table, ids, kept)
            dy, dtable = ops.linear_distillation_backward(dloss, y, table, ids, kept, lse)
            dq, dk, dv, _ = ops.linear_attention_backward(dy.view_as(out), None, x, x, x, decay)
            ops.embedding_backward((dq + dk + dv).view_as(y), words, vocab, dweight=dtable, accumulate=True)
            step = ops.linear_attention_step(x[:, :, 0], x[:, :, 0], x[:, :, 0], decay, state)
            return loss, dtable, state, step

        return call

    users = [user(1, 2, 3000, 128, 2, 4, 300, 7), user(2, 1, 5000, 240, 4, 3, 700, 33)]
    want = [call() for call in users]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in users]
    got = [[], []]
    for _ in range(10):
        for i, call in enumerate(users):
            with torch.cuda.stream(streams[i]):
                got[i].append(call())
    for stream in streams:
        with torch.cuda.stream(stream):
            ops.check()
    torch.cuda.synchronize()
    for i in range(2):
        for results in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(results, want[i]))
