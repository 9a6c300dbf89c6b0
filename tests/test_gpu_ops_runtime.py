"""The training operators around their arithmetic: waits that run out, CUDA graphs, offsets past 32 bits, calls in a row."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    from paper_1810_07766_b200 import build, ops

    build.build()
    return ops


@pytest.mark.parametrize("n,tokens,outs,cols", [(1, 64, 300, 260), (2, 700, 100, 64), (1, 5000, 1000, 700)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_wait_that_runs_out_is_reported(ops, dtype, n, tokens, outs, cols):
    """No copies are issued, so the kernel's waits for data give up after 200 ms; it ends by itself and the next check says so.  After that
    the same call works."""
    lib = ops._library()
    dy = torch.randn(n, tokens, outs, device="cuda").to(dtype)
    packed = ops.pack_activation(torch.randn(n, tokens, cols, device="cuda").to(dtype))
    want = ops.packed_weight_grad(dy, packed)
    ops.check()
    out = torch.full_like(want, 7.0)
    d = ops.rps_wgrad_desc(dtype=ops._DTYPE[dtype], n=n, tokens=tokens, outs=outs, cols=cols, dy_row=outs, dy_worker=tokens * outs, dweight_row=cols,
                           dweight_worker=outs * cols, wait_limit_ms=200, withhold_copies=1)
    size = ctypes.c_size_t()
    assert lib.rps_wgrad_workspace(ctypes.byref(d), dy.data_ptr(), ctypes.byref(size)) == 0
    ws = torch.zeros(size.value, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    assert lib.rps_packed_wgrad(ctypes.byref(d), dy.data_ptr(), packed.codes.data_ptr(), packed.scales.data_ptr(), out.data_ptr(), ws.data_ptr(),
                                size.value, stream) == 0
    with pytest.raises(ops.RPSError, match="gave up"):
        ops.check()
    ops.check()      # reported once
    again = ops.packed_weight_grad(dy, packed)
    ops.check()
    assert torch.equal(again, want)


def test_calls_in_a_cuda_graph(ops):
    n, T, V, D = 2, 200, 700, 96
    g = torch.Generator(device="cuda").manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    x, f, w = r(n, T, D), r(n, T, D), r(n, V, D) / 10
    gate, post, pre, dh = r(n, 1, D), r(n, D), r(n, D), r(n, T, D)
    y = torch.randint(0, V, (n, T), generator=g, device="cuda")
    dloss = torch.ones(n, device="cuda")

    def step():
        h, out, kept = ops.gated_residual_norm_forward(x, f, gate, post, pre, keep="int8")
        loss, lse = ops.linear_cross_entropy_forward(out, w, y)
        dy, dw = ops.linear_cross_entropy_backward(dloss, out, w, y, lse)
        grads = ops.gated_residual_norm_backward(dh, dy, kept, gate, post, pre)
        return (loss, dw, ops.packed_weight_grad(grads[1], kept.h)) + grads

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in (1, 2):
        g.manual_seed(seed)
        for t in (x, f):
            t.copy_(r(*t.shape))
        y.copy_(torch.randint(0, V, (n, T), generator=g, device="cuda"))
        y[0, :seed * 20] = -100
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, step()):
            assert torch.equal(a, b)


def test_activations_past_32_bit_offsets(ops):
    """2^31 elements and more: the last rows come out as those of a small call."""
    rows, cols = 270_000, 8192
    x = torch.zeros(1, rows, cols, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(0)
    tail = torch.randn(1, 3, cols, generator=g, device="cuda").bfloat16()
    x[:, -3:] = tail
    p, q = ops.pack_activation(x), ops.pack_activation(tail)
    assert torch.equal(p.codes[:, -3:], q.codes) and torch.equal(p.scales[:, -3:], q.scales)
    assert not p.codes[:, :-3].any()
    back = ops.unpack_activation(p)
    assert torch.equal(back[:, -3:], ops.unpack_activation(q))
    del back, p
    ones = torch.ones(1, cols, dtype=torch.bfloat16, device="cuda")
    gate = ones[:, None] * 0.5
    h, y, kept = ops.gated_residual_norm_forward(x, x, gate, ones, ones, keep="int8")
    hs, ys, small = ops.gated_residual_norm_forward(tail, tail, gate, ones, ones, keep="int8")
    assert torch.equal(h[:, -3:], hs) and torch.equal(y[:, -3:], ys) and torch.equal(kept.h.codes[:, -3:], small.h.codes)
    dx, df, dgate, dpost, dpre = ops.gated_residual_norm_backward(None, y, kept, gate, ones, ones)
    sx, sf, sgate, spost, spre = ops.gated_residual_norm_backward(None, ys, small, gate, ones, ones)
    assert torch.equal(dx[:, -3:], sx) and torch.equal(df[:, -3:], sf) and not dx[:, :-3].any()
    for a, b in ((dgate, sgate), (dpost, spost), (dpre, spre)):   # the other rows add zeros
        assert torch.allclose(a.float(), b.float(), rtol=2 ** -7, atol=2.0 ** -14)


def test_many_different_calls_in_a_row(ops):
    """Nothing of a call is left for the next one: results of a mixed sequence are those of the calls made alone."""
    g = torch.Generator(device="cuda").manual_seed(3)
    calls = []
    for n, T, V, D, dtype in ((1, 5, 40, 33, torch.float32), (3, 300, 500, 64, torch.bfloat16), (2, 129, 257, 130, torch.float32), (4, 1, 1000, 24, torch.bfloat16)):
        h = torch.randn(n, T, D, generator=g, device="cuda").to(dtype)
        w = torch.randn(n, V, D, generator=g, device="cuda").to(dtype) / 4
        y = torch.randint(0, V, (n, T), generator=g, device="cuda")
        calls.append((h, w, y))

    def run(c):
        loss, lse = ops.linear_cross_entropy_forward(*c)
        return (loss, lse) + ops.linear_cross_entropy_backward(torch.ones_like(loss), *c, lse)

    alone = []
    for c in calls:
        alone.append(run(c))
        torch.cuda.synchronize()
    for _ in range(3):
        together = [run(c) for c in calls * 2]
        torch.cuda.synchronize()
        for got, want in zip(together, alone * 2):
            assert all(torch.equal(a, b) for a, b in zip(got, want))
