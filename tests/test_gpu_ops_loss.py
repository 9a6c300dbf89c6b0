"""The linear cross entropy against its definition in 64 bits.

Tolerances, from the number formats.  e16 = 2^-8 is half a unit of bf16's last place, e32 = 2^-23 one of fp32's (sums may be
cut off instead of rounded).
  logits    |error| <= (6 cols + 16) e32 * A, A = sum |h| |w| of the largest logit: one addition of fp32 each, six products
            for the three parts of an fp32 value
  p         a relative error of twice that, and 2^-20 for exp and its argument
  gradients the same relative error for each term, e16 more where dl is rounded to bf16; terms summed in fp32; one rounding to the
            result's type
so an element is held to  (relative error of a term) * (sum of the terms' sizes) + (rounding of the result)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

E16, E32 = 2.0 ** -8, 2.0 ** -23
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    from paper_1810_07766_b200 import build, ops

    build.build()
    return ops


def inputs(dtype, n, T, V, D, ignored=0.0, seed=0, spread=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn(n, T, D, generator=g, device="cuda").to(TYPES[dtype])
    w = (torch.randn(n, V, D, generator=g, device="cuda") * spread / D ** 0.5).to(TYPES[dtype])
    y = torch.randint(0, V, (n, T), generator=g, device="cuda")
    y[torch.rand(n, T, generator=g, device="cuda") < ignored] = -100
    return h, w, y


def definition(h, w, y, dloss, reduction, ignore=-100):
    """loss, lse, dhidden, dweight in 64 bits and, for the tolerance, the sums of the terms' sizes."""
    n, T, D = h.shape
    out = {"lse": torch.zeros(n, T), "each": torch.zeros(n, T), "dh": torch.zeros(n, T, D), "dw": torch.zeros(w.shape), "sh": torch.zeros(n, T, D),
           "sw": torch.zeros(w.shape), "loss": torch.zeros(n, T) if reduction == "none" else torch.zeros(n)}
    out = {k: v.double().cuda() for k, v in out.items()}
    out["size"] = 0.0
    for i in range(n):
        keep = torch.nonzero(y[i] != ignore).flatten()
        m = len(keep)
        if m == 0:
            continue
        hi, wi, yi, k = h[i, keep].double(), w[i].double(), y[i, keep], torch.arange(m, device="cuda")
        z = hi @ wi.T
        out["size"] = max(out["size"], float((hi.abs() @ wi.abs().T).max()))
        lse = torch.logsumexp(z, 1)
        each = lse - z[k, yi]
        out["lse"][i, keep], out["each"][i, keep] = lse, each
        g = (dloss[i, keep] if reduction == "none" else dloss[i].expand(m)).double() / (m if reduction == "mean" else 1)
        p = torch.exp(z - lse[:, None]) * g[:, None]
        q = p.abs()
        p[k, yi] -= g
        q[k, yi] += g.abs()
        out["dh"][i, keep], out["dw"][i] = p @ wi, p.T @ hi
        out["sh"][i, keep], out["sw"][i] = q @ wi.abs(), q.T @ hi.abs()
        if reduction != "none":
            out["loss"][i] = each.sum() / (m if reduction == "mean" else 1)
    if reduction == "none":
        out["loss"] = out["each"]
    return out


def check(ops, dtype, h, w, y, reduction="mean", dloss=None, dweight=None, run=None):
    n, T, D = h.shape
    V = w.shape[1]
    if dloss is None:
        g = torch.Generator(device="cuda").manual_seed(5)
        dloss = torch.rand((n, T) if reduction == "none" else (n,), generator=g, device="cuda") + 0.5
    loss, lse = ops.linear_cross_entropy_forward(h, w, y, reduction=reduction)
    dh, dw = ops.linear_cross_entropy_backward(dloss, h, w, y, lse, reduction=reduction, dweight=dweight)
    torch.cuda.synchronize()
    want = definition(h, w, y, dloss, reduction)
    logit = (6 * D + 16) * E32 * want["size"]
    scale = T if reduction == "sum" else 1
    assert ((lse - want["lse"]).abs() <= logit + 2.0 ** -20 * (1 + want["lse"].abs())).all()
    assert ((loss - want["loss"]).abs() <= scale * (2 * logit + 2.0 ** -20 * (2 + want["lse"].abs().max()))).all()
    half = dtype == "bf16"
    term = 2 * logit + 2.0 ** -20 + (E16 if half else 0.0)
    for got, name, size, terms in ((dh, "dh", "sh", V), (dw, "dw", "sw", T)):
        assert got.dtype == TYPES[dtype] and got.shape == want[name].shape
        bound = (term + (6 * terms + 16) * E32) * want[size] + (E16 if half else E32) * want[name].abs()
        assert ((got - want[name]).abs() <= bound).all(), (name, float(((got - want[name]).abs() - bound).max()))
        # errors of independent roundings: a whole gradient is nearer than its elements' bounds say
        norm = want[name].norm()
        assert (got - want[name]).norm() <= (5e-3 if half else 1e-5) * norm + 1e-300, (name, float((got - want[name]).norm() / norm))
    assert (dh[y == -100] == 0).all() and (lse[y == -100] == 0).all()
    return loss, lse, dh, dw


SIZES = [(1, 1, 1, 1), (1, 1, 2, 3), (2, 3, 5, 7), (1, 64, 64, 64), (1, 65, 129, 65), (3, 130, 257, 100), (1, 257, 300, 72), (2, 300, 1000, 33),
         (4, 32, 1000, 256), (1, 1, 5000, 520), (1, 1000, 17, 130), (64, 5, 40, 16), (1, 513, 769, 1025)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,T,V,D", SIZES)
def test_sizes(ops, dtype, n, T, V, D):
    check(ops, dtype, *inputs(dtype, n, T, V, D))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
@pytest.mark.parametrize("ignored", [0.3, 0.99])
def test_reductions_and_ignored_tokens(ops, dtype, reduction, ignored):
    h, w, y = inputs(dtype, 3, 200, 333, 48, ignored=ignored, seed=3)
    y[1] = -100            # a worker none of whose tokens takes part
    h[:, :, :][y == -100] = float("nan")   # what ignored rows hold is not read
    h[0, :2][y[0, :2] == -100] = float("inf")
    loss, lse, dh, dw = check(ops, dtype, h, w, y, reduction=reduction)
    assert (loss[1] == 0).all() and (dw[1] == 0).all() and (dh[1] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_other_ignore_index_and_no_tokens(ops, dtype):
    h, w, y = inputs(dtype, 2, 20, 30, 16)
    loss, lse = ops.linear_cross_entropy_forward(h, w, y, ignore_index=7, reduction="none")
    assert ((loss == 0) == (y == 7)).all() or (y == 7).sum() == 0
    for reduction in ("none", "sum", "mean"):
        loss, lse = ops.linear_cross_entropy_forward(h[:, :0], w, y[:, :0], reduction=reduction)
        assert loss.shape == ((2, 0) if reduction == "none" else (2,)) and (loss == 0).all() and lse.shape == (2, 0)
        dh, dw = ops.linear_cross_entropy_backward(torch.ones_like(loss), h[:, :0], w, y[:, :0], lse, reduction=reduction,
                                                   dweight=torch.full_like(w, float("nan")))
        assert dh.shape == (2, 0, 16) and (dw == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_target_that_names_no_row_poisons_its_worker_alone(ops, dtype):
    h, w, y = inputs(dtype, 2, 20, 30, 16)
    for bad in (30, -1, 1 << 40):
        y[1, 4] = bad
        loss, lse = ops.linear_cross_entropy_forward(h, w, y)
        dh, dw = ops.linear_cross_entropy_backward(torch.ones(2, device="cuda"), h, w, y, lse)
        assert torch.isfinite(loss[0]) and torch.isnan(loss[1])
        assert torch.isfinite(dw[0]).all() and torch.isnan(dw[1]).all() and torch.isnan(dh[1, 4]).all()
        each, _ = ops.linear_cross_entropy_forward(h, w, y, reduction="none")
        assert torch.isnan(each).sum() == 1 and torch.isnan(each[1, 4])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_parameters_out_of_a_replica_array(ops, dtype, offset):
    """Weights are views into the rows of an [n][pitch] array, at any offset, and so may the gradient be."""
    n, T, V, D = 3, 70, 90, 24
    h, w, y = inputs(dtype, n, T, V, D, seed=8)
    pitch = 256 * 10
    flat = torch.full((n, pitch), float("nan"), dtype=TYPES[dtype], device="cuda")
    grad = torch.full((n, pitch), 7.0, dtype=TYPES[dtype], device="cuda")
    view = lambda a: a[:, offset:offset + V * D].view(n, V, D)  # noqa: E731
    view(flat).copy_(w)
    _, _, _, dw = check(ops, dtype, h, view(flat), y, dweight=view(grad))
    assert dw.data_ptr() == view(grad).data_ptr()
    assert (grad[:, :offset] == 7).all() and (grad[:, offset + V * D:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_rows_and_a_shared_weight(ops, dtype):
    n, T, V, D = 2, 50, 60, 40
    h, w, y = inputs(dtype, n, T, V, D, seed=9)
    wide = torch.full((n, T, D + 9), float("nan"), dtype=h.dtype, device="cuda")
    wide[:, :, 1:D + 1] = h
    rows = torch.full((n, V, D + 5), float("nan"), dtype=h.dtype, device="cuda")
    rows[:, :, :D] = w
    out = torch.full((n, V, D + 3), 7.0, dtype=h.dtype, device="cuda")
    check(ops, dtype, wide[:, :, 1:D + 1], rows[:, :, :D], y, dweight=out[:, :, :D])
    assert (out[:, :, D:] == 7).all()
    # one weight for all workers (stride 0): a gradient for each; workers interleaved in the gradient
    out = torch.full((V, n, D), 7.0, dtype=h.dtype, device="cuda")
    check(ops, dtype, h, w[:1].expand(n, V, D), y, dweight=out.transpose(0, 1))


@pytest.mark.parametrize("dtype,n,T,V,D", [("f32", 8, 200, 30000, 16), ("bf16", 16, 250, 40000, 24)])
def test_more_than_one_piece_of_the_vocabulary(ops, dtype, n, T, V, D):
    check(ops, dtype, *inputs(dtype, n, T, V, D, ignored=0.2, seed=4))


def test_large_logits(ops):
    """Logits of some hundreds: the running maximum keeps the exponentials in range."""
    for dtype in ("f32", "bf16"):
        h, w, y = inputs(dtype, 1, 100, 300, 64, spread=150.0)
        loss, lse = ops.linear_cross_entropy_forward(h, w, y, reduction="none")
        want = definition(h, w, y, torch.ones(1, 100, device="cuda"), "none")
        assert want["lse"].abs().max() > 300
        tol = (6 * 64 + 16) * E32 * want["size"] * 2 + 2.0 ** -20 * (1 + want["lse"].abs().max())
        assert ((loss - want["loss"]).abs() <= tol).all()
        dh, dw = ops.linear_cross_entropy_backward(torch.ones(1, 100, device="cuda"), h, w, y, lse, reduction="none")
        assert torch.isfinite(dh).all() and torch.isfinite(dw).all()


def test_weights_past_32_bit_offsets(ops):
    V, D, T = 270_000, 8192, 3
    w = torch.zeros(1, V, D, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    w[0, -5:] = (torch.randn(5, D, generator=g, device="cuda") / 64).bfloat16()
    h = torch.randn(1, T, D, generator=g, device="cuda").bfloat16()
    y = torch.tensor([[V - 1, 0, V - 4]], device="cuda")
    loss, lse = ops.linear_cross_entropy_forward(h, w, y, reduction="none")
    z = h[0].double() @ w[0, -5:].double().T
    want = torch.log(torch.exp(z).sum(1) + (V - 5))
    assert torch.allclose(lse[0].double(), want, atol=1e-4, rtol=0)
    hit = torch.stack([z[0, 4], torch.zeros((), device="cuda", dtype=torch.float64), z[2, 1]])
    assert torch.allclose(loss[0].double(), want - hit, atol=2e-4, rtol=0)
    dh, dw = ops.linear_cross_entropy_backward(torch.ones_like(loss), h, w, y, lse, reduction="none")
    p = torch.exp(z - want[:, None])
    p[0, 4] -= 1
    p[2, 1] -= 1
    assert (dw[0, -5:].double() - p.T @ h[0].double()).norm() <= 5e-3 * (p.T @ h[0].double()).norm()
    assert (dh[0].double() - p @ w[0, -5:].double()).norm() <= 5e-3 * (p @ w[0, -5:].double()).norm()
    rest = torch.exp(-want)
    first = rest[0] * h[0, 0].double() + (rest[1] - 1) * h[0, 1].double() + rest[2] * h[0, 2].double()
    assert (dw[0, 0].double() - first).norm() <= 5e-3 * first.norm()


def test_gradient_against_differences(ops):
    """Central differences of the kernel's own loss along the gradient: with a step s the quotient is off by O(s^2) of the third
    derivative and by the loss's fp32 error over s.  Loss about 6 with an error below 2^-20 * 8; s * |grad| = 0.1."""
    h, w, y = inputs("f32", 1, 80, 150, 32, ignored=0.2)
    hh, ww = h.clone().requires_grad_(), w.clone().requires_grad_()
    ops.linear_cross_entropy(hh, ww, y).sum().backward()
    for name, at, grad in (("hidden", h, hh.grad), ("weight", w, ww.grad)):
        size = float(grad.norm())
        step = grad / size * (0.02 / size)
        f = lambda v: float(ops.linear_cross_entropy_forward(*((v, w) if name == "hidden" else (h, v)), y)[0])  # noqa: E731
        quotient = (f(at + step) - f(at - step)) / 2
        assert quotient == pytest.approx(0.02, rel=2e-2), name


def test_autograd_matches_the_direct_calls(ops):
    h, w, y = inputs("bf16", 2, 60, 100, 32, ignored=0.2)
    hh, ww = h.clone().requires_grad_(), w.clone().requires_grad_()
    loss = ops.linear_cross_entropy(hh, ww, y, reduction="none")
    loss.sum().backward()      # an expanded gradient
    l0, lse = ops.linear_cross_entropy_forward(h, w, y, reduction="none")
    dh, dw = ops.linear_cross_entropy_backward(torch.ones_like(l0), h, w, y, lse, reduction="none")
    assert torch.equal(loss, l0) and torch.equal(hh.grad, dh) and torch.equal(ww.grad, dw)
    # without the worker axis
    one = ops.linear_cross_entropy(h[1], w[1], y[1], reduction="none")
    assert torch.equal(one, l0[1])


def test_same_inputs_same_bits_on_any_stream(ops):
    h, w, y = inputs("bf16", 2, 300, 700, 64, ignored=0.2)
    first = check(ops, "bf16", h, w, y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = check(ops, "bf16", h, w, y)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(first, again):
        assert torch.equal(a, b)


def test_refusals(ops):
    h, w, y = inputs("bf16", 2, 8, 10, 16)
    bad = [(h.half(), w.half(), y), (h, w.float(), y), (h, w, y.int()), (h, w, y[:, :4]), (h, w[:1], y), (h, w[:, :, :8], y), (h[0], w, y),
           (h.transpose(1, 2), w, y), (h, w, y.cpu()), (h, w.cpu(), y), (h[0, 0], w[0, 0], y[0])]
    for a in bad:
        with pytest.raises(ValueError):
            ops.linear_cross_entropy_forward(*a)
    with pytest.raises(ValueError):
        ops.linear_cross_entropy_forward(h, w, y, reduction="avg")
    loss, lse = ops.linear_cross_entropy_forward(h, w, y)
    for dloss, l in ((torch.ones(3, device="cuda"), lse), (torch.ones(2, device="cuda").double(), lse), (torch.ones(2, device="cuda"), lse[:, :4])):
        with pytest.raises(ValueError):
            ops.linear_cross_entropy_backward(dloss, h, w, y, l)
    with pytest.raises(ops.RPSError):
        ops.linear_cross_entropy_backward(torch.ones(2, device="cuda"), h, w, y, lse, dweight=torch.empty_like(w[:1]).expand(2, 10, 16))
    with pytest.raises(ops.RPSError):
        ops.linear_cross_entropy_forward(h[:, :, :0], w[:, :, :0], y)
