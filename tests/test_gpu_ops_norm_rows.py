"""The norms with many rows to a CTA and to a cluster: slots of the ring used again, sums exchanged in both rooms and both phases, workers and
gate groups that begin in the middle of a CTA's rows.  The bounds are those of test_gpu_ops_norm_pack.py."""
import pytest
import torch

from test_gpu_ops_norm_pack import check_norm, norm_inputs, ops  # noqa: F401

pytestmark = pytest.mark.gpu

# Rows over clusters of 2 to 8 CTAs, whole and ragged last slices; each cluster has 3 to 15 of them.
CLUSTERS = [("f32", 1, 1200, 2052, 1), ("f32", 2, 301, 4096, 7), ("f32", 3, 200, 4488, 1), ("f32", 1, 600, 5400, 300), ("f32", 1, 500, 6148, 1),
            ("f32", 2, 130, 8192, 1), ("f32", 1, 300, 10243, 4), ("f32", 1, 220, 12300, 1), ("f32", 2, 60, 16384, 60), ("bf16", 1, 1100, 4104, 1),
            ("bf16", 2, 350, 5001, 1), ("bf16", 3, 200, 8200, 2), ("bf16", 1, 400, 12298, 1), ("bf16", 2, 120, 16384, 10)]
# Rows of one CTA each: more than the ring's four slots, at each of the three alignments; the workers' rows end inside a CTA's.
CTAS = [("f32", 3, 700, 2048, 1), ("f32", 3, 1100, 1001, 1100), ("f32", 5, 2500, 250, 10), ("f32", 3, 9500, 64, 1), ("bf16", 3, 700, 4096, 7),
        ("bf16", 3, 700, 4095, 1), ("bf16", 3, 1100, 2002, 2), ("bf16", 5, 2000, 333, 2000), ("bf16", 3, 9500, 85, 1), ("bf16", 7, 1500, 1000, 3)]


@pytest.mark.parametrize("keep", ["values", "int8"])
@pytest.mark.parametrize("dtype,n,T,D,gates", CLUSTERS + CTAS)
def test_many_rows(ops, dtype, n, T, D, gates, keep):  # noqa: F811
    s = norm_inputs(dtype, n, T, D, gates, seed=D)
    first = check_norm(ops, dtype, s, keep=keep)
    ops.check()
    again = ops.gated_residual_norm_forward(s["x"], s["f"], s["gate"], s["post"], s["pre"], scale=0.7, eps=1e-5, keep=keep)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    grads = ops.gated_residual_norm_backward(s["dh"], s["dy"], again[2], s["gate"], s["post"], s["pre"], scale=0.7)
    assert all(torch.equal(a, b) for a, b in zip(first[2:], grads))


@pytest.mark.parametrize("dtype,n,T,D", [("f32", 2, 400, 4490), ("bf16", 2, 400, 5002), ("f32", 2, 900, 1003), ("bf16", 2, 900, 2050)])
def test_many_rows_without_a_gradient_of_h(ops, dtype, n, T, D):  # noqa: F811
    check_norm(ops, dtype, norm_inputs(dtype, n, T, D, 1, seed=D), use_dh=False)
