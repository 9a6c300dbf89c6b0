"""Linear attention at the ends of what it takes: infinities among bf16 operands."""
import pytest
import torch

from test_gpu_ops_attention import inputs, ops, definition, run  # noqa: F401

pytestmark = pytest.mark.gpu

CHUNK = 128   # tokens of the longest chunk: what is further apart than that meets through a state


def kind(t):
    """0: finite, 1: infinite, -1: minus infinity, 2: NaN."""
    return torch.where(torch.isnan(t), 2, torch.where(torch.isinf(t), torch.sign(t), 0.0).to(torch.int64))


@pytest.mark.parametrize("mixed", [False, True])
@pytest.mark.parametrize("T,H,K,W", [(400, 3, 64, 64), (400, 3, 128, 128), (3000, 2, 40, 72), (180, 3, 33, 31), (120, 3, 100, 127), (400, 3, 20, 77)])
def test_an_infinity_goes_through_states(ops, T, H, K, W, mixed):  # noqa: F811
    """One infinity in each of several heads of sequences, of operands of one sign or of both.  States, and results that lie in other chunks, are finite,
    infinite or NaN as the definition's; in its own chunk what the definition makes infinite or NaN is one of these; all other heads keep their bits.
    Sequences for the tensor cores' both kernels, in segments, and by way of copies."""
    n, B, t = 1, 6, T // 2 if T < 1000 else 2100
    x = inputs("bf16", n, B, T, H, K, W, seed=T + K)
    x["log_decay"].fill_(-0.02)
    for name in ("q", "k", "v", "dout"):
        x[name] = torch.where(x[name] == 0, 1.0, x[name]).to(torch.bfloat16)
    if not mixed:
        x = {name: a if name == "log_decay" else a.abs() for name, a in x.items()}
    clean = run(ops, x, 0.5)
    x["v"][0, 0, t, 0, 3], x["k"][0, 1, t, 1, 2], x["q"][0, 2, t, 0, 4], x["dout"][0, 3, t, 1, 5] = float("inf"), -float("inf"), -float("inf"), float("inf")
    x["v"][0, 4, t, 1, 6], x["k"][0, 4, t, 1, 1] = -float("inf"), 0.0   # a zero meets it
    x["q"][0, 5, t, 0, 7], x["dout"][0, 5, t, 0, 0] = float("inf"), float("inf")
    got, want = run(ops, x, 0.5), definition(x, 0.5)
    touched = {(0, 0), (1, 1), (2, 0), (3, 1), (4, 1), (5, 0)}
    far = (torch.arange(T, device="cuda") - t).abs() >= CHUNK
    for name in got:
        for s in range(B):
            for h in range(H):
                pick = (lambda a: a[0, s, h]) if "state" in name else (lambda a: a[0, s, :, h])  # noqa: E731
                mine, other = pick(got[name]), pick(want[name])
                if (s, h) not in touched:
                    assert torch.equal(mine, pick(clean[name])), (name, s, h)
                    continue
                if "state" in name:
                    assert torch.equal(kind(mine), kind(other)), (name, s, h)
                    fine = torch.isfinite(other)
                    assert (mine[fine] - other[fine]).norm() <= 5e-6 * other[fine].norm(), (name, s, h)
                else:
                    assert torch.equal(kind(mine[far]), kind(other[far])), (name, s, h)
                    assert not (torch.isfinite(mine) & ~torch.isfinite(other)).any(), (name, s, h)
    # one of q is in its own token's result alone
    rows = torch.arange(T, device="cuda") != t
    assert torch.equal(got["out"][0, 2, rows, 0], clean["out"][0, 2, rows, 0]) and torch.equal(got["state"][0, 2, 0], clean["state"][0, 2, 0])
