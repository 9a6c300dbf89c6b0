"""Distillation from a teacher's kept logits against its definition in 64 bits.

Tolerances, from the number formats, as those of the cross entropy.  e16 = 2^-8 is half a step of bf16, e32 = 2^-23 a step of fp32 (sums may be cut
off instead of rounded), tau the temperature.
  logits    |error| <= (6 cols + 16) e32 * A, A the largest sum |h| |w|
  p, q      relative errors of 2 / tau times that and 2^-20 for exp and its argument; q 2^-20 alone
  lse       that of the logits and 2^-20 (tau + |lse|)
  loss      tau^2 sum q (log q - log p): tau times the logits' errors, and 2^-20 of its terms' sizes
  gradients those relative errors for each term, e16 more where dl is rounded to bf16; terms summed in fp32; one rounding of the result"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

E16, E32 = 2.0 ** -8, 2.0 ** -23
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
IGNORE = -100


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    from paper_1810_07766_b200 import build, ops

    build.build()
    return ops


def inputs(dtype, n, T, V, D, top, seed=0, ignored=0.0, spread=2.0, logits="f32"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn(n, T, D, generator=g, device="cuda").to(TYPES[dtype])
    w = (torch.randn(n, V, D, generator=g, device="cuda") * spread / D ** 0.5).to(TYPES[dtype])
    ids = torch.randint(0, V, (n, T, top), generator=g, device="cuda")      # words may come twice
    x = (torch.randn(n, T, top, generator=g, device="cuda") * 3).to(TYPES[logits])
    ids[torch.rand(n, T, top, generator=g, device="cuda") < 0.2] = IGNORE
    ids[torch.rand(n, T, generator=g, device="cuda") < ignored] = IGNORE
    return h, w, ids, x


def definition(h, w, ids, x, tau, dloss, reduction, ignore=IGNORE):
    n, T, D = h.shape
    V = w.shape[1]
    out = {"lse": torch.zeros(n, T), "each": torch.zeros(n, T), "se": torch.zeros(n, T), "dh": torch.zeros(n, T, D), "dw": torch.zeros(w.shape),
           "sh": torch.zeros(n, T, D), "sw": torch.zeros(w.shape), "loss": torch.zeros(n, T) if reduction == "none" else torch.zeros(n),
           "sl": torch.zeros(n, T) if reduction == "none" else torch.zeros(n)}
    out = {k: v.double().cuda() for k, v in out.items()}
    out["size"], out["valid"] = 0.0, ((ids != ignore) & (x > -math.inf)).any(-1)
    for i in range(n):
        keep = torch.nonzero(out["valid"][i]).flatten()
        m = len(keep)
        if m == 0:
            continue
        hi, wi = h[i, keep].double(), w[i].double()
        at = ids[i, keep]
        y = torch.where(at == ignore, -math.inf, x[i, keep].double() / tau)
        q = torch.softmax(y, -1)
        log_q = torch.where(q > 0, torch.log_softmax(y, -1), 0.0)
        at = torch.where(q > 0, at, 0)
        z = hi @ wi.T
        out["size"] = max(out["size"], float((hi.abs() @ wi.abs().T).max()))
        lse = torch.logsumexp(z / tau, 1) * tau
        log_p = (z - lse[:, None]).gather(1, at) / tau
        out["lse"][i, keep] = lse
        out["each"][i, keep] = tau ** 2 * (q * (log_q - log_p)).sum(1)
        out["se"][i, keep] = tau ** 2 * (q * (log_q.abs() + log_p.abs() + (lse[:, None] / tau).abs() + 1)).sum(1)
        g = (dloss[i, keep] if reduction == "none" else dloss[i].expand(m)).double() / (m if reduction == "mean" else 1) * tau
        p = torch.exp((z - lse[:, None]) / tau)
        size = p.scatter_add(1, at, q) * g.abs()[:, None]
        p = p.scatter_add(1, at, -q) * g[:, None]
        out["dh"][i, keep], out["dw"][i] = p @ wi, p.T @ hi
        out["sh"][i, keep], out["sw"][i] = size @ wi.abs(), size.T @ hi.abs()
        if reduction != "none":
            by = m if reduction == "mean" else 1
            out["loss"][i], out["sl"][i] = out["each"][i].sum() / by, out["se"][i].sum() / by
    if reduction == "none":
        out["loss"], out["sl"] = out["each"], out["se"]
    return out


def check(ops, dtype, h, w, ids, x, tau=1.0, reduction="mean", dweight=None):
    n, T, D = h.shape
    V = w.shape[1]
    g = torch.Generator(device="cuda").manual_seed(5)
    dloss = torch.rand((n, T) if reduction == "none" else (n,), generator=g, device="cuda") + 0.5
    loss, lse = ops.linear_distillation_forward(h, w, ids, x, temperature=tau, reduction=reduction)
    dh, dw = ops.linear_distillation_backward(dloss, h, w, ids, x, lse, temperature=tau, reduction=reduction, dweight=dweight)
    torch.cuda.synchronize()
    want = definition(h, w, ids, x, tau, dloss, reduction)
    logit = (6 * D + 16) * E32 * want["size"]
    many = T if reduction == "sum" else 1
    assert ((lse - want["lse"]).abs() <= logit + 2.0 ** -20 * (tau + want["lse"].abs())).all()
    assert ((loss - want["loss"]).abs() <= 2 * tau * logit * many + 2.0 ** -20 * want["sl"]).all(), float(((loss - want["loss"]).abs()).max())
    half = dtype == "bf16"
    term = 2 * logit / tau + 2.0 ** -19 + (E16 if half else 0.0)
    for got, name, size, terms in ((dh, "dh", "sh", V), (dw, "dw", "sw", T)):
        assert got.dtype == TYPES[dtype] and got.shape == want[name].shape
        bound = (term + (6 * terms + 16) * E32) * want[size] + (E16 if half else E32) * want[name].abs()
        assert ((got - want[name]).abs() <= bound).all(), (name, float(((got - want[name]).abs() - bound).max()))
        # errors of independent roundings: a whole gradient is nearer than its elements' bounds say (p - q may be smaller than both)
        assert (got - want[name]).norm() <= (5e-3 if half else 1e-5) * want[size].norm() + 1e-300, name
    assert (dh[~want["valid"]] == 0).all() and (lse[~want["valid"]] == 0).all()
    return loss, lse, dh, dw


SIZES = [(1, 1, 1, 1, 1), (1, 1, 2, 3, 4), (2, 3, 5, 7, 2), (1, 64, 64, 64, 8), (1, 65, 129, 65, 33), (3, 130, 257, 100, 64), (1, 257, 300, 72, 65), (2, 300, 1000, 33, 10),
         (4, 32, 1000, 256, 100), (1, 1, 5000, 520, 256), (1, 1000, 17, 130, 129), (64, 5, 40, 16, 3), (1, 513, 769, 1025, 20)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,T,V,D,top", SIZES)
def test_sizes(ops, dtype, n, T, V, D, top):
    check(ops, dtype, *inputs(dtype, n, T, V, D, top, seed=T, logits="bf16" if T % 2 else "f32"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,T,V,D,top", [(1, 1, 20000, 300, 40), (2, 2, 1000, 2049, 5), (8, 3, 5000, 64, 256), (3, 4, 777, 130, 100), (1, 5, 9000, 96, 64), (2, 8, 3000, 200, 33),
                                         (1, 9, 3000, 200, 33)])
def test_a_few_tokens(ops, dtype, n, T, V, D, top):
    """Up to four of bf16 and eight of fp32 go through dot products; some without entries, words in the same entries, the vocabulary's first and last."""
    h, w, ids, x = inputs(dtype, n, T, V, D, top, seed=T)
    ids[:, :, 0], ids[:, :, 1], ids[:, :, 2] = V - 1, 0, V - 1
    check(ops, dtype, h, w, ids, x, tau=1.5)
    ids[-1, T // 2] = IGNORE
    h[-1, T // 2] = float("nan")
    for reduction in ("none", "sum"):
        check(ops, dtype, h, w, ids, x, tau=0.7, reduction=reduction)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_few_tokens_with_mistakes(ops, dtype):
    h, w, ids, x = inputs(dtype, 2, 3, 50, 16, 4, seed=1)
    ids[1, 2, 1] = 50
    loss, lse = ops.linear_distillation_forward(h, w, ids, x)
    dh, dw = ops.linear_distillation_backward(torch.ones(2, device="cuda"), h, w, ids, x, lse)
    assert torch.isfinite(loss[0]) and torch.isnan(loss[1]) and torch.isfinite(dh[0]).all() and torch.isfinite(dw[0]).all()
    assert torch.isnan(dh[1, 2]).all() and torch.isnan(dw[1]).all() and torch.isfinite(dh[1, :2]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
@pytest.mark.parametrize("tau", [0.5, 3.0])
def test_reductions_temperatures_and_tokens_without_entries(ops, dtype, reduction, tau):
    h, w, ids, x = inputs(dtype, 3, 200, 333, 48, 12, ignored=0.4, seed=3)
    ids[1] = IGNORE                                  # a worker none of whose tokens takes part
    x[2, :50] = -math.inf                            # tokens with words that the teacher rules out
    x[2, 50:100, 1:] = -math.inf                     # one word left (or none)
    none = ((ids == IGNORE) | (x == -math.inf)).all(-1)
    h[none] = float("nan")                           # not read
    h[0, :2][none[0, :2]] = float("inf")
    loss, lse, dh, dw = check(ops, dtype, h, w, ids, x, tau=tau, reduction=reduction)
    assert (loss[1] == 0).all() and (dw[1] == 0).all() and (dh[1] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_word_is_the_cross_entropy(ops, dtype):
    """A teacher that is sure of one word has no entropy of its own: loss and gradients are those of the cross entropy, up to both sides'
    roundings (held to the definition by their own tests: here twice that of a p)."""
    h, w, ids, x = inputs(dtype, 2, 150, 400, 40, 1, ignored=0.2, seed=4)
    loss, lse, dh, dw = check(ops, dtype, h, w, ids, x)
    want, other = ops.linear_cross_entropy_forward(h, w, ids[..., 0])
    assert torch.equal(lse, other) and ((loss - want).abs() <= 2.0 ** -18 * (1 + want)).all()
    a, b = ops.linear_cross_entropy_backward(torch.ones_like(loss), h, w, ids[..., 0], other)
    c, d = ops.linear_distillation_backward(torch.ones_like(loss), h, w, ids, x, lse)
    assert torch.equal(a, c) and torch.equal(b, d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_all_words_kept_and_words_kept_twice(ops, dtype):
    """Every word of the vocabulary in a random order, each token's in another; and one word in all entries."""
    n, T, V = 2, 70, 200
    h, w, ids, x = inputs(dtype, n, T, V, 40, V, seed=5)
    ids = torch.rand(n, T, V, device="cuda").argsort(-1)
    check(ops, dtype, h, w, ids, x, tau=2.0)
    check(ops, dtype, h, w, ids // 7 * 7, x)
    check(ops, dtype, h, w, torch.full_like(ids, V - 1), x)


def test_a_student_that_is_its_teacher(ops):
    """Nothing to learn: loss and gradients vanish but for roundings, whose sizes the definition's terms give."""
    h, w, _, _ = inputs("f32", 1, 50, 180, 32, 1, seed=6)
    x, ids = torch.topk((h.double() @ w.double().mT).float(), 180)
    loss, lse, dh, dw = check(ops, "f32", h, w, ids, x, tau=1.5)
    assert float(loss) <= 1e-4


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_mistakes_poison_their_worker_alone(ops, dtype):
    h, w, ids, x = inputs(dtype, 2, 20, 30, 16, 4)
    cases = []
    for bad in (30, -1, 1 << 40):
        i = ids.clone()
        i[1, 4, 2] = bad
        cases.append((i, x))
    for bad in (float("nan"), float("inf")):
        i, y = ids.clone(), x.clone()
        i[1, 4, 2], y[1, 4, 2] = 3, bad
        cases.append((i, y))
    for i, y in cases:
        loss, lse = ops.linear_distillation_forward(h, w, i, y)
        dh, dw = ops.linear_distillation_backward(torch.ones(2, device="cuda"), h, w, i, y, lse)
        assert torch.isfinite(loss[0]) and torch.isnan(loss[1])
        assert torch.isfinite(dh[0]).all() and torch.isfinite(dw[0]).all() and torch.isnan(dh[1, 4]).all() and torch.isnan(dw[1]).all()
        each, _ = ops.linear_distillation_forward(h, w, i, y, reduction="none")
        assert torch.isnan(each[1, 4]) and torch.isnan(each).sum() == 1
    # NaN in an entry that is none is nothing
    i, y = ids.clone(), x.clone()
    i[1, 4, 2], y[1, 4, 2] = IGNORE, float("nan")
    assert torch.isfinite(ops.linear_distillation_forward(h, w, i, y)[0]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [3, 300])
@pytest.mark.parametrize("spread", [1e6, 1e15])
def test_logits_of_any_size(ops, dtype, T, spread):
    h, w, ids, x = inputs(dtype, 2, T, 500, 48, 6, seed=T, spread=spread)
    loss, lse, dh, dw = check(ops, dtype, h, w, ids, x)
    assert torch.isfinite(loss).all() and torch.isfinite(dh).all() and torch.isfinite(dw).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_tokens_and_another_ignore_index(ops, dtype):
    h, w, ids, x = inputs(dtype, 2, 20, 30, 16, 5)
    for reduction in ("none", "sum", "mean"):
        loss, lse = ops.linear_distillation_forward(h[:, :0], w, ids[:, :0], x[:, :0], reduction=reduction)
        assert loss.shape == ((2, 0) if reduction == "none" else (2,)) and (loss == 0).all() and lse.shape == (2, 0)
        dh, dw = ops.linear_distillation_backward(torch.ones_like(loss), h[:, :0], w, ids[:, :0], x[:, :0], lse, reduction=reduction,
                                                  dweight=torch.full_like(w, float("nan")))
        assert dh.shape == (2, 0, 16) and (dw == 0).all()
    a = ops.linear_distillation_forward(h, w, ids, x, reduction="none")[0]
    b = ops.linear_distillation_forward(h, w, torch.where(ids == IGNORE, 7, torch.where(ids == 7, IGNORE, ids)), x, ignore_index=7, reduction="none")[0]
    without = (ids != 7).all(-1)
    assert torch.equal(a[without], b[without]) and torch.isnan(b[~without]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parameters_and_gradients_in_rows_of_a_larger_array(ops, dtype):
    n, T, V, D = 3, 80, 90, 40
    h, w, ids, x = inputs(dtype, n, T, V, D, 9)
    for shift in (0, 1, 8):
        flat = torch.full((n, shift + 2 * V * D + 24), 7.0, device="cuda").to(TYPES[dtype])
        weight = flat[:, shift:shift + V * D].view(n, V, D)
        weight.copy_(w)
        out = flat[:, shift + V * D:shift + 2 * V * D].view(n, V, D)
        hidden = torch.zeros(n, T, D + shift, device="cuda").to(TYPES[dtype])[..., shift:].copy_(h)
        wide = torch.stack([x, x], -1)[..., 0]
        check(ops, dtype, hidden, weight, ids.transpose(0, 1).contiguous().transpose(0, 1), wide, dweight=out)
        assert (flat[:, :shift] == 7).all() and (flat[:, shift + 2 * V * D:] == 7).all() and torch.equal(weight, w)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_vocabulary_in_pieces(ops, dtype):
    """So large that it goes through in several pieces, with entries on both sides of each border."""
    T, V, D, top = (2048, 140_000, 32, 16) if dtype == "bf16" else (1000, 100_000, 24, 16)
    h, w, ids, x = inputs(dtype, 1, T, V, D, top, seed=8)
    ids[0, ::3, 0] = torch.arange(len(ids[0, ::3]), device="cuda") * 256 % V
    ids[0, ::3, 1] = (torch.arange(len(ids[0, ::3]), device="cuda") * 256 + 255) % V
    ids[0, ::2, 2], ids[0, ::2, 3] = V - 1, 0
    check(ops, dtype, h, w, ids, x, tau=2.0)


def test_through_autograd_and_without_a_worker_axis(ops):
    h, w, ids, x = inputs("bf16", 2, 60, 100, 32, 7, ignored=0.3)
    a, b = h.clone().requires_grad_(), w.clone().requires_grad_()
    loss = ops.linear_distillation(a, b, ids, x, temperature=2.0)
    (loss * torch.tensor([1.0, 3.0], device="cuda")).sum().backward()
    want, lse = ops.linear_distillation_forward(h, w, ids, x, temperature=2.0)
    dh, dw = ops.linear_distillation_backward(torch.tensor([1.0, 3.0], device="cuda"), h, w, ids, x, lse, temperature=2.0)
    assert torch.equal(loss, want) and torch.equal(a.grad, dh) and torch.equal(b.grad, dw)
    assert torch.equal(ops.linear_distillation(h[1], w[1], ids[1], x[1], temperature=2.0), want[1])


def test_gradients_of_differences(ops):
    """Central differences of the loss along random directions: off by their third-order term (a step of 2^-7 of logits that spread by
    2: below 2^-10 of the product) and the loss's roundings over the step."""
    h, w, ids, x = inputs("f32", 1, 40, 60, 24, 6, seed=9)
    loss = lambda a, b: ops.linear_distillation_forward(a, b, ids, x, temperature=1.5)[0].double()  # noqa: E731
    value, lse = ops.linear_distillation_forward(h, w, ids, x, temperature=1.5)
    dh, dw = ops.linear_distillation_backward(torch.ones(1, device="cuda"), h, w, ids, x, lse, temperature=1.5)
    size = 2.0 ** -7
    for leaf, grad in ((h, dh), (w, dw)):
        step = grad / grad.norm()   # along the gradient, so that the product is its norm
        change = (loss(h + size * step, w) - loss(h - size * step, w) if leaf is h else loss(h, w + size * step) - loss(h, w - size * step)) / (2 * size)
        rounding = 2.0 ** -20 * (1 + float(value)) / size
        assert abs(float(change) - float(grad.norm())) <= 2.0 ** -9 * float(grad.norm()) + rounding


def test_arguments_are_refused(ops):
    h, w, ids, x = inputs("f32", 2, 10, 8, 16, 4)
    lse, dloss = torch.zeros(2, 10, device="cuda"), torch.zeros(2, device="cuda")
    f, b = ops.linear_distillation_forward, ops.linear_distillation_backward
    many = torch.zeros(2, 10, 257, dtype=torch.int64, device="cuda")
    for call, match in ((lambda: f(h.cpu(), w, ids, x), "CUDA"), (lambda: f(h, w[:1], ids, x), "weight must have shape"), (lambda: f(h, w.bfloat16(), ids, x), "type"),
                        (lambda: f(h, w, ids.int(), x), "top_ids must be"), (lambda: f(h, w, ids[:, :9], x), "top_ids must be"), (lambda: f(h, w, ids[..., 0], x), "top_ids must be"),
                        (lambda: f(h, w, ids, x[..., :3]), "top_logits must have shape"), (lambda: f(h, w, ids, x.half()), "float32 or bfloat16"),
                        (lambda: f(h, w, ids, x, temperature=0.0), "temperature"), (lambda: f(h, w, ids, x, temperature=float("nan")), "temperature"),
                        (lambda: f(h, w, ids, x, temperature=-1.0), "temperature"), (lambda: f(h, w, ids, x, reduction="max"), "reduction"),
                        (lambda: f(h, w, ids[..., :0], x[..., :0]), "top"), (lambda: f(h, w, many, many.float()), "256"), (lambda: f(h.mT, w, ids, x), "shape|contiguous"),
                        (lambda: b(dloss[:1], h, w, ids, x, lse), "dloss must be"), (lambda: b(dloss, h, w, ids, x, lse[:, :9]), "lse must be"),
                        (lambda: b(dloss, h, w, ids, x, lse, dweight=w[:, :7]), "dweight must have shape"),
                        (lambda: ops.linear_distillation(h, w, ids, x.requires_grad_()), "no gradient")):
        with pytest.raises((ValueError, ops.RPSError), match=match):
            call()


def test_the_same_bits_every_time_in_graphs_and_on_other_streams(ops):
    h, w, ids, x = inputs("bf16", 2, 300, 700, 96, 10)
    dloss = torch.ones(2, device="cuda")

    def step():
        loss, lse = ops.linear_distillation_forward(h, w, ids, x, temperature=2.0)
        return (loss, lse) + ops.linear_distillation_backward(dloss, h, w, ids, x, lse, temperature=2.0)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in (1, 2):
        for mine, other in zip((h, w, ids, x), inputs("bf16", 2, 300, 700, 96, 10, seed=seed, ignored=0.1 * seed)):
            mine.copy_(other)
        graph.replay()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = step()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(held, again))
    ops.check()
