"""A wait for another CTA's sums that runs out, in the norms of rows that several CTAs share."""
import ctypes

import pytest
import torch

from test_gpu_ops_norm_pack import TYPES, norm_inputs, ops  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,n,T,D", [("f32", 1, 4, 4096), ("f32", 2, 150, 5200), ("bf16", 1, 300, 16384)])  # clusters of 2 to 5, one row and many
def test_a_wait_that_runs_out_is_reported(ops, dtype, n, T, D):  # noqa: F811
    """One CTA of each row sends no sums: the others' waits give up after 20 ms, the kernels end by themselves, write nothing of the rows and the
    next check says so.  After that the same calls work."""
    lib = ops._library()
    s = norm_inputs(dtype, n, T, D, 1, seed=D)
    a = [s[k] for k in ("x", "f", "gate", "post", "pre")]
    at = lambda *tensors: [t.data_ptr() for t in tensors]  # noqa: E731
    h, y, kept = ops.gated_residual_norm_forward(*a)
    grads = ops.gated_residual_norm_backward(s["dh"], s["dy"], kept, *a[2:])
    ops.check()
    d = ops.rps_norm_desc(dtype=ops._DTYPE[TYPES[dtype]], n=n, tokens=T, cols=D, gates=1, post_worker=D, pre_worker=D, gate_worker=D, scale=1.0, eps=1e-6,
                          wait_limit_ms=20, withhold_sums=1)
    stream = torch.cuda.current_stream().cuda_stream
    out = [torch.full_like(h, 7.0), torch.full_like(y, 7.0)]
    r = torch.full_like(kept.r, 7.0)
    assert lib.rps_norm_forward(ctypes.byref(d), *at(*a, *out, r[0], r[1]), None, None, None, None, stream) == 0
    with pytest.raises(ops.RPSError, match="gave up"):
        ops.check()
    assert all((t == 7).all() for t in out) and (r == 7).all()
    ops.check()      # reported once
    size = ctypes.c_size_t()
    assert lib.rps_norm_workspace(ctypes.byref(d), ctypes.byref(size)) == 0
    ws = torch.zeros(size.value, dtype=torch.uint8, device="cuda")
    void = [torch.full_like(g, 7.0) for g in grads]
    args = at(s["dh"], s["dy"], s["f"]) + [None] + at(h) + [None] + at(kept.r_f, kept.r_h, *a[2:], *void, ws)
    assert lib.rps_norm_backward(ctypes.byref(d), *args, size.value, stream) == 0
    with pytest.raises(ops.RPSError, match="gave up"):
        ops.check()
    assert all((t == 7).all() for t in void[:2])
    ops.check()
    h2, y2, again = ops.gated_residual_norm_forward(*a)
    assert torch.equal(h2, h) and torch.equal(y2, y)
    assert all(torch.equal(u, v) for u, v in zip(grads, ops.gated_residual_norm_backward(s["dh"], s["dy"], again, *a[2:])))
    ops.check()
