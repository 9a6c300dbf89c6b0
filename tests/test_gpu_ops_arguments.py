"""Arguments of the training operators that are neither plain numbers nor of one shape."""
import pytest
import torch

from test_gpu_ops_norm_pack import norm_inputs, ops  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("device", ["cpu", "cuda"])
def test_a_scale_that_changes_between_calls(ops, device):  # noqa: F811
    """A number held in a tensor is read in every call: what is kept of a call goes by values."""
    s = norm_inputs("f32", 1, 8, 40, 1)
    a = [s[k] for k in ("x", "f", "gate", "post", "pre")]
    scale, eps = torch.tensor(0.5, device=device), torch.tensor(1e-6, device=device)
    for value, small in ((0.5, 1e-6), (2.0, 1e-6), (2.0, 0.25)):
        scale.fill_(value), eps.fill_(small)
        h, y, kept = ops.gated_residual_norm_forward(*a, scale=scale, eps=eps)
        wh, wy, want = ops.gated_residual_norm_forward(*a, scale=float(scale), eps=float(eps))
        assert torch.equal(h, wh) and torch.equal(y, wy)
        got = ops.gated_residual_norm_backward(s["dh"], s["dy"], kept, *a[2:], scale=scale)
        for u, v in zip(got, ops.gated_residual_norm_backward(s["dh"], s["dy"], want, *a[2:], scale=float(scale))):
            assert torch.equal(u, v)


def test_a_scale_that_changes_before_the_backward_pass(ops):  # noqa: F811
    s = norm_inputs("f32", 1, 8, 40, 1)
    grads = []
    for change in (False, True):
        scale = torch.tensor(0.5)
        leaves = [s[k].clone().requires_grad_() for k in ("x", "f", "gate", "post", "pre")]
        h, y = ops.gated_residual_norm(*leaves, scale=scale)
        if change:
            scale.fill_(3.0)
        (h * s["dh"] + y * s["dy"]).sum().backward()
        grads.append([v.grad for v in leaves])
    assert all(torch.equal(a, b) for a, b in zip(*grads))


def test_a_scale_that_wants_a_gradient_is_refused(ops):  # noqa: F811
    s = norm_inputs("f32", 1, 8, 40, 1)
    with pytest.raises(ValueError, match="scale"):
        ops.gated_residual_norm(*(s[k] for k in ("x", "f", "gate", "post", "pre")), scale=torch.tensor(0.5, requires_grad=True))


@pytest.mark.parametrize("x,weight", [((1, 5, 8), (2, 6, 8)), ((2, 5, 8), (1, 6, 8)), ((5, 8), (6, 9)), ((2, 5, 8), (3, 6, 8))])
def test_linear_8bit_of_shapes_that_do_not_go_together(ops, x, weight):  # noqa: F811
    """Refused before the product, not at its gradient."""
    with pytest.raises(ValueError, match="weight"):
        ops.linear_8bit(torch.ones(x, device="cuda"), torch.ones(weight, device="cuda"))


def test_linear_8bit_of_two_types_or_places(ops):  # noqa: F811
    x, w = torch.ones(5, 8, device="cuda"), torch.ones(6, 8, device="cuda")
    for a, b in ((x.bfloat16(), w), (x, w.bfloat16()), (x.double(), w.double()), (x, w.cpu()), (x.cpu(), w)):
        with pytest.raises(ValueError):
            ops.linear_8bit(a, b)
