"""The linear cross entropy of a few tokens, whose logits are dot products instead of tensor-core tiles: the same definition and
bounds (sums of fp32 products in fp32 lie well inside those of the other path), across both ends of the token counts."""
import pytest
import torch

from test_gpu_ops_loss import TYPES, check, inputs, ops  # noqa: F401

pytestmark = pytest.mark.gpu

SIZES = [(1, 1, 1, 1), (2, 1, 7, 3), (1, 2, 33, 8), (3, 2, 500, 333), (2, 3, 1000, 520), (1, 4, 4001, 1300), (5, 4, 77, 129), (2, 5, 300, 100),
         (1, 7, 1025, 1001), (4, 8, 2000, 256), (2, 9, 300, 100), (64, 3, 40, 16), (64, 1, 513, 64), (1, 1, 20000, 4100),
         (1, 4, 300, 6401), (1, 2, 300, 12801), (1, 1, 60, 25601), (1, 8, 300, 3201)]  # the last ones: one column more than is held


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,T,V,D", SIZES)
def test_sizes(ops, dtype, n, T, V, D):  # noqa: F811
    check(ops, dtype, *inputs(dtype, n, T, V, D, seed=T + V))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
@pytest.mark.parametrize("T", [1, 3, 4, 8])
def test_reductions_and_ignored_tokens(ops, dtype, reduction, T):  # noqa: F811
    h, w, y = inputs(dtype, 4, T, 333, 48, ignored=0.4, seed=3)
    y[1] = -100
    y[2, 0] = -100
    h[y == -100] = float("nan")
    loss, lse, dh, dw = check(ops, dtype, h, w, y, reduction=reduction)
    assert (loss[1] == 0).all() and (dw[1] == 0).all() and (dh[1] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 4])
def test_a_target_that_names_no_row_poisons_its_worker_alone(ops, dtype, T):  # noqa: F811
    h, w, y = inputs(dtype, 2, T, 30, 16)
    for bad in (30, -1, 1 << 40):
        y[1, T - 1] = bad
        loss, lse = ops.linear_cross_entropy_forward(h, w, y)
        dh, dw = ops.linear_cross_entropy_backward(torch.ones(2, device="cuda"), h, w, y, lse)
        assert torch.isfinite(loss[0]) and torch.isnan(loss[1])
        assert torch.isfinite(dw[0]).all() and torch.isnan(dw[1]).all() and torch.isnan(dh[1, T - 1]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [0, 1, 2, 3])
@pytest.mark.parametrize("T", [1, 4])
def test_parameters_out_of_a_replica_array(ops, dtype, offset, T):  # noqa: F811
    n, V, D = 3, 90, 40
    h, w, y = inputs(dtype, n, T, V, D, seed=8)
    pitch = 256 * 15
    flat = torch.full((n, pitch), float("nan"), dtype=TYPES[dtype], device="cuda")
    grad = torch.full((n, pitch), 7.0, dtype=TYPES[dtype], device="cuda")
    view = lambda a, o: a[:, o:o + V * D].view(n, V, D)  # noqa: E731
    view(flat, offset).copy_(w)
    other = 8 if offset == 2 else offset  # aligned gradients of weights that are not, too
    check(ops, dtype, h, view(flat, offset), y, dweight=view(grad, other))
    assert (grad[:, :other] == 7).all() and (grad[:, other + V * D:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_rows_and_a_shared_weight(ops, dtype):  # noqa: F811
    n, T, V, D = 2, 4, 60, 40
    h, w, y = inputs(dtype, n, T, V, D, seed=9)
    wide = torch.full((n, T, D + 9), float("nan"), dtype=h.dtype, device="cuda")
    wide[:, :, 1:D + 1] = h
    rows = torch.full((n, V, D + 5), float("nan"), dtype=h.dtype, device="cuda")
    rows[:, :, :D] = w
    out = torch.full((n, V, D + 3), 7.0, dtype=h.dtype, device="cuda")
    check(ops, dtype, wide[:, :, 1:D + 1], rows[:, :, :D], y, dweight=out[:, :, :D])
    assert (out[:, :, D:] == 7).all()
    out = torch.full((V, n, D), 7.0, dtype=h.dtype, device="cuda")
    check(ops, dtype, h, w[:1].expand(n, V, D), y, dweight=out.transpose(0, 1))


def test_weights_past_32_bit_offsets(ops):  # noqa: F811
    """A weight of 2^31 elements and more: its last rows alone are not zero, so the definition needs them alone."""
    V, D, tail = (1 << 20) + 700, 2056, 500
    w = torch.zeros(1, V, D, dtype=torch.bfloat16, device="cuda")
    h, small, y = inputs("bf16", 1, 2, tail, D, seed=11)
    w[:, V - tail:] = small
    y += V - tail
    loss, lse = ops.linear_cross_entropy_forward(h, w, y)
    dh, dw = ops.linear_cross_entropy_backward(torch.ones(1, device="cuda"), h, w, y, lse)
    logits = h[0].double() @ small[0].double().T
    want = torch.logsumexp(torch.cat([logits, torch.full((2, 1), torch.log(torch.tensor(float(V - tail))).item(), device="cuda").double()], 1), 1)
    assert ((lse[0] - want).abs() <= 1e-4 * want).all()
    p = torch.exp(logits - want[:, None])
    p[torch.arange(2), y[0] - (V - tail)] -= 1
    got, exact = dw[0, V - tail:].double(), (p / 2).T @ h[0].double()
    assert (got - exact).norm() <= 5e-3 * exact.norm()
    exact = (p / 2) @ small[0].double()
    assert (dh[0] - exact).norm() <= 5e-3 * exact.norm()
    rest = torch.exp(-want).sum().item() / 2 * h.abs().max().item()
    assert dw[0, :V - tail].abs().max().item() <= rest * 1.01


@pytest.mark.parametrize("dtype,T", [("f32", 1), ("f32", 8), ("bf16", 1), ("bf16", 4)])
def test_same_inputs_same_bits(ops, dtype, T):  # noqa: F811
    h, w, y = inputs(dtype, 2, T, 3000, 203, seed=2)
    first = check(ops, dtype, h, w, y)
    again = check(ops, dtype, h, w, y)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
