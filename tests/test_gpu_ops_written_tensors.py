"""Tensors of the caller's that a call writes to: autograd knows that they have changed."""
import pytest
import torch

from test_gpu_ops_attention import ops  # noqa: F401

pytestmark = pytest.mark.gpu


def writers(ops):  # noqa: F811
    """Calls that write to a dweight [6, 8]."""
    h, w, y = torch.randn(5, 8, device="cuda"), torch.randn(6, 8, device="cuda"), torch.tensor([0, 5, 2, 2, 1], device="cuda")
    ids, kept, one = y[:, None].contiguous(), torch.zeros(5, 1, device="cuda"), torch.ones((), device="cuda")
    _, lse = ops.linear_distillation_forward(h, w, ids, kept)
    return {"distillation": lambda d: ops.linear_distillation_backward(one, h, w, ids, kept, lse, dweight=d),
            "embedding": lambda d: ops.embedding_backward(h, y, 6, dweight=d),
            "embedding, added": lambda d: ops.embedding_backward(h, y, 6, dweight=d, accumulate=True)}


@pytest.mark.parametrize("name", ["distillation", "embedding", "embedding, added"])
def test_a_gradient_that_needs_the_old_values_says_so(ops, name):  # noqa: F811
    write = writers(ops)[name]
    d = torch.randn(6, 8, device="cuda")
    factor = torch.randn(6, 8, device="cuda", requires_grad=True)
    product = (factor * d).sum()          # keeps d for factor's gradient
    before = d._version
    write(d)
    assert d._version > before
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        product.backward()


def test_a_step_takes_no_new_state_that_wants_a_gradient_and_changes_none_that_it_did_not_write(ops, monkeypatch):  # noqa: F811
    B, H, K = 2, 2, 8
    q, k, v = (torch.randn(B, H, K, device="cuda") for _ in "qkv")
    ld, state, other = torch.full((H,), -0.1, device="cuda"), torch.randn(B, H, K, K, device="cuda"), torch.zeros(B, H, K, K, device="cuda")
    leaf = torch.zeros_like(state, requires_grad=True)
    with pytest.raises(ValueError, match="new_state"):
        ops.linear_attention_step(q, k, v, ld, state, new_state=leaf)
    assert leaf._version == 0 and not leaf.any()
    with torch.no_grad():
        ops.linear_attention_step(q, k, v, ld, state, new_state=leaf)
    assert leaf._version == 1 and leaf.any()

    def fails(*args):
        raise ops.RPSError(-3, "rps_linear_attention_step", "it failed")

    before = state._version, other._version
    monkeypatch.setattr(ops, "_call", fails)
    for new in (None, other):
        with pytest.raises(ops.RPSError):
            ops.linear_attention_step(q, k, v, ld, state, new_state=new)
    assert (state._version, other._version) == before
