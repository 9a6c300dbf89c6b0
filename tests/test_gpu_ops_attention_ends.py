"""Linear attention at the ends of what it takes: infinities among bf16 operands, long sequences under a short limit on waits,
hundreds of lengths."""
import pytest
import torch

from test_gpu_ops_attention import check, definition, inputs, ops, run  # noqa: F401

pytestmark = pytest.mark.gpu

CHUNK = 128   # tokens of the longest chunk: what is further apart than that meets through a state


def kind(t):
    """0: finite, 1: infinite, -1: minus infinity, 2: NaN."""
    return torch.where(torch.isnan(t), 2, torch.where(torch.isinf(t), torch.sign(t), 0.0).to(torch.int64))


@pytest.mark.parametrize("mixed", [False, True])
@pytest.mark.parametrize("T,H,K,W", [(400, 3, 64, 64), (400, 3, 128, 128), (3000, 2, 40, 72), (180, 3, 33, 31), (120, 3, 100, 127), (400, 3, 20, 77)])
def test_an_infinity_goes_through_states(ops, T, H, K, W, mixed, dtype="bf16"):  # noqa: F811
    """One infinity in each of several heads of sequences, of operands of one sign or of both.  States, and results that lie in other chunks, are finite,
    infinite or NaN as the definition's; in its own chunk what the definition makes infinite or NaN is one of these; all other heads keep their bits.
    Sequences for the tensor cores' both kernels, in segments, and by way of copies."""
    n, B, t = 1, 6, T // 2 if T < 1000 else 2100
    x = inputs(dtype, n, B, T, H, K, W, seed=T + K)
    x["log_decay"].fill_(-0.02)
    x["log_decay"][:, 1] = 0.0   # whose powers leave an operand's few bits as they are
    for name in ("q", "k", "v", "dout"):
        x[name] = torch.where(x[name] == 0, torch.ones_like(x[name]), x[name])
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


@pytest.mark.parametrize("T,H,K,W", [(400, 3, 64, 64), (3000, 2, 40, 72), (180, 3, 33, 31)])
def test_an_infinity_goes_through_states_in_fp32(ops, T, H, K, W):  # noqa: F811
    for mixed in (False, True):
        test_an_infinity_goes_through_states(ops, T, H, K, W, mixed, "f32")


@pytest.mark.parametrize("backward", [False, True])
def test_a_limit_on_waits_is_none_on_sequences(ops, backward):  # noqa: F811
    """Sequences that a CTA takes several times longer for than its waits for data may last: 1875 chunks of 2.8 us against 2 ms.  Nothing gives up, and
    results are those of the default limit."""
    import ctypes

    T, H, K = 240_000, 300, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(1, T, H, K, generator=g, device="cuda", dtype=torch.bfloat16) for _ in "qkv")
    ld = torch.full((H,), -0.05, device="cuda")
    rest = {"scale": 0.5}
    want = ops.linear_attention_backward(v, None, q, k, v, ld, **rest) if backward else ops.linear_attention_forward(q, k, v, ld, **rest)
    ops.check()
    s = ops.rps_axis_strides(0, T * H * K, H * K, K)
    d = ops.rps_linear_attention_desc(dtype=1, n=1, heads=H, wait_limit_ms=2, sequences=1, tokens=T, key_cols=K, value_cols=K, q=s, k=s, v=s, dout=s, scale=0.5)
    size, lib = ctypes.c_size_t(), ops._library()
    assert lib.rps_linear_attention_workspace(ctypes.byref(d), int(backward), ctypes.byref(size)) == 0 and size.value == 0   # no segments
    got = [torch.full_like(t, float("nan")) for t in want]
    p = [t.data_ptr() for t in got]
    stream = torch.cuda.current_stream().cuda_stream
    if backward:
        status = lib.rps_linear_attention_backward(ctypes.byref(d), v.data_ptr(), None, q.data_ptr(), k.data_ptr(), v.data_ptr(), ld.data_ptr(), None, None, *p, None, 0, stream)
    else:
        status = lib.rps_linear_attention_forward(ctypes.byref(d), q.data_ptr(), k.data_ptr(), v.data_ptr(), ld.data_ptr(), None, None, *p, None, 0, stream)
    assert status == 0
    ops.check()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_heads_without_columns_are_refused(ops):  # noqa: F811
    x = inputs("f32", 1, 2, 5, 3, 4, 8)
    q, v, ld, s = x["q"][..., :0], x["v"], x["log_decay"], x["state"][..., :0, :].contiguous()
    for call in (lambda: ops.linear_attention(q, q, v, ld), lambda: ops.linear_attention_forward(q, q, v, ld), lambda: ops.linear_attention_backward(v, None, q, q, v, ld),
                 lambda: ops.linear_attention_step(q[:, :, 0], q[:, :, 0], v[:, :, 0], ld, s)):
        with pytest.raises(ops.RPSError, match="key_cols"):
            call()
    with pytest.raises(ValueError, match="q must be"):
        ops.linear_attention(q.sum(), q, v, ld)


@pytest.mark.parametrize("n,B", [(4, 64), (1, 257), (2, 129)])
def test_sequences_of_many_lengths(ops, n, B):  # noqa: F811
    """Up to 256 sequences are taken the longest first, more as they come; several have the same length."""
    x = inputs("bf16", n, B, 140, 2, 32, 24, seed=B)
    lengths = torch.randint(-1, 142, (n, B), generator=torch.Generator(device="cuda").manual_seed(B), device="cuda")
    lengths[:, ::5] = 130
    check(ops, x, lengths=lengths)


@pytest.mark.parametrize("n,B,T,H,K,W", [(1, 40, 8, 8, 64, 64), (2, 3, 64, 5, 16, 48), (1, 2, 150, 3, 64, 8), (3, 7, 192, 2, 40, 64), (1, 5, 1, 4, 8, 8)])
def test_short_sequences_of_narrow_heads_at_any_address(ops, n, B, T, H, K, W):  # noqa: F811
    """They go through the kernel of short chunks however they lie, so that their results do not depend on it."""
    x = inputs("bf16", n, B, T, H, K, W, seed=T)
    want, y = check(ops, x), dict(x)
    for name in ("q", "k", "v", "dout"):
        room = torch.zeros(x[name].numel() + 1, dtype=torch.bfloat16, device="cuda")[1:].view_as(x[name])
        y[name] = room.copy_(x[name])
    got = run(ops, y, 0.3)
    assert all(torch.equal(got[name], want[name]) for name in want)


def test_offsets_past_32_bits_in_short_sequences(ops):  # noqa: F811
    """2^31 elements and more in every tensor, states among them.  Heads that forget at once: each result is its own token's."""
    B, T, H, D = 262_400, 64, 2, 64
    x = torch.zeros(B, T, H, D, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(T, H, D, device="cuda").bfloat16()
    x[-1] = tail
    never = torch.full((H,), float("-inf"), device="cuda")
    t = tail.double()
    want = t.square().sum(-1, keepdim=True) * t
    last = t[-1, :, :, None] * t[-1, :, None, :]
    out, state = ops.linear_attention_forward(x, x, x, never, scale=1.0)
    assert state.numel() > 2 ** 31 and not out[:-1].any() and (out[-1] - want).norm() <= 5e-3 * want.norm()
    assert not state[:-1].any() and (state[-1] - last).norm() <= 5e-6 * last.norm()
    del out, state
    dq, dk, dv, first = ops.linear_attention_backward(x, None, x, x, x, never, scale=1.0)
    for grad in (dq, dk, dv):
        assert not grad[:-1].any() and (grad[-1] - want).norm() <= 5e-3 * want.norm()
    assert not first.any()
