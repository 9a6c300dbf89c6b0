"""Distillation at the ends of its range: the hottest and coldest temperatures, logits that are large next to their differences.

Logits here are sums of few numbers of few bits, so that neither side rounds them.  What remains, from the number formats, with tau the temperature:
  loss      tau^2 sum q (log(q sum) + (top - l) / tau): q and the sum of exponentials are off by 2^-21 and 2^-20 (exponentials 2^-22, their sums over tiles),
            the difference of logits by a rounding or two: tau^2 (2^-19 + 2^-22 times its terms)
  p         exp((l - lse) / tau), lse one fp32 number: 2^-23 |lse| / tau (its sum's rounding and its own), and 2^-19
  gradients those of p and q for each term, 2^-8 more with bf16, terms summed in fp32, one rounding of the result; as a whole, since one element's
            p - q may be smaller than either"""
import pytest
import torch

from test_gpu_ops_distillation import TYPES, definition, ops  # noqa: F401

pytestmark = pytest.mark.gpu


def exact(dtype, n, T, V, top, shift=0.0, seed=0):
    """Logits of shift and a multiple of 1/8 between -14 and 14; the first two words have the same."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randint(-1, 2, (n, T, 8), generator=g, device="cuda").float()
    w = torch.randint(-16, 17, (n, V, 8), generator=g, device="cuda").float() / 8
    h[..., 0], w[..., 0] = 1.0, shift
    w[:, 1] = w[:, 0]
    ids = torch.rand(n, T, V, generator=g, device="cuda").argsort(-1)[..., :top].contiguous()
    x = torch.randn(n, T, top, generator=g, device="cuda")
    return h.to(TYPES[dtype]), w.to(TYPES[dtype]), ids, x


def check(ops, dtype, h, w, ids, x, tau):  # noqa: F811
    n, T = h.shape[:2]
    dloss = torch.ones(n, T, device="cuda")
    loss, lse = ops.linear_distillation_forward(h, w, ids, x, temperature=tau, reduction="none")
    dh, dw = ops.linear_distillation_backward(dloss, h, w, ids, x, lse, temperature=tau, reduction="none")
    want = definition(h, w, ids, x, tau, dloss, "none")
    off = (loss - want["loss"]).abs() - (tau ** 2 * 2.0 ** -19 + 2.0 ** -22 * want["sl"])
    assert (off <= 0).all(), float(off.max())
    p = 2.0 ** -23 * float(want["lse"].abs().max()) / tau + 2.0 ** -19 + (2.0 ** -8 if dtype == "bf16" else 0.0)
    for got, name, size in ((dh, "dh", "sh"), (dw, "dw", "sw")):
        assert (got - want[name]).norm() <= p * want[size].norm(), (name, float((got - want[name]).norm() / want[size].norm()), p)
    return loss, lse, dh, dw


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [3, 70])
@pytest.mark.parametrize("tau", [0.01, 100.0])
def test_the_coldest_and_the_hottest(ops, dtype, T, tau):  # noqa: F811
    """Through dot products and tiles.  Where two words share all the probability, what the gradient takes from them and gives to the teacher's words
    adds up to nothing."""
    h, w, ids, x = exact(dtype, 2, T, 300, 200, seed=T)
    check(ops, dtype, h, w, ids, x * tau, tau)
    w[:, 2:] /= 2
    w[:, :2, 1:] = 0
    w[:, :2, 0], w[:, 2:, 0] = 16.0, 0.0
    loss, lse, dh, dw = check(ops, dtype, h, w, ids, x * tau, tau)
    if dtype == "f32":
        assert (dw[..., 0].sum(1).abs() <= T * tau * (2.0 ** -23 * 32 / tau + 2.0 ** -19)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [3, 300])
def test_logits_all_larger_by_a_number(ops, dtype, T):  # noqa: F811
    """It changes neither probabilities nor losses, and so not what the losses are off by: no term of them is as large as the logits are."""
    tau = 1.0
    h, w, ids, x = exact(dtype, 2, T, 300, 40, shift=1024.0, seed=T)
    loss, lse = ops.linear_distillation_forward(h, w, ids, x, temperature=tau, reduction="none")
    want = definition(h, w, ids, x, tau, torch.ones(2, T, device="cuda"), "none")
    terms = want["sl"] - tau * (want["lse"].abs() + tau)     # without lse's
    off = (loss - want["loss"]).abs() - (tau ** 2 * 2.0 ** -19 + 2.0 ** -22 * terms)
    assert (off <= 0).all(), float(off.max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [3, 70])
def test_teachers_whose_logits_are_large_next_to_their_differences(ops, dtype, T):  # noqa: F811
    """Differences that fp32 holds exactly are what probabilities are made of, and infinite ones of finite logits are certainty."""
    h, w, ids, x = exact(dtype, 2, T, 300, 20, seed=T)
    x = 32768.0 + torch.arange(20, device="cuda") / 256 + torch.zeros_like(x)
    check(ops, dtype, h, w, ids, x, 0.01)
    x[..., 7], x[..., 9] = 3e38, -3e38
    loss, lse, dh, dw = check(ops, dtype, h, w, ids, x, 0.01)
    assert torch.isfinite(loss).all() and torch.isfinite(dw).all()
    x[:] = -3e38
    check(ops, dtype, h, w, ids, x, 0.01)
