"""Linear attention with a decay for each head against its recurrence in 64 bits, token by token.

Tolerances, from the number formats.  `size` is a result made of the sizes of all inputs, so the sum of the sizes of its terms.
  bf16 results  masked scores and states are rounded to bf16 where they are multiplied once more: each term once, by 2^-8 at most; one
                rounding of the result; fp32 sums below that
  fp32 results  and states: each term in the three parts that stand for fp32 values, which leave out 6 * 2^-24, and a decay rounded to
                fp32 twice
  fp32 sums     may be cut off instead of rounded, 2^-23 a step: 6 products for every 16 of the summed axes (cols, 64 tokens, cols), one step for each
                chunk, two for each segment
  fp32's end    a decay's power or a term below 2^-126 may count as zero: at most 2^26 (tokens * cols * sizes) of those to a result
Whole results are nearer than their elements' bounds say, as the errors are of independent roundings: 5e-3 (bf16), 5e-6 (fp32, states)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    from paper_1810_07766_b200 import build, ops

    build.build()
    return ops


def inputs(dtype, n, B, T, H, K, W, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = {"q": r(n, B, T, H, K), "k": r(n, B, T, H, K), "v": r(n, B, T, H, W), "dout": r(n, B, T, H, W)}
    x = {name: t.to(TYPES[dtype]) for name, t in x.items()}
    x["log_decay"] = torch.log1p(-torch.exp2(-1.0 - 8.0 * torch.rand(n, H, generator=g, device="cuda")))
    x["state"], x["dstate"] = r(n, B, H, K, W), r(n, B, H, K, W)
    return x


def definition(x, scale, lengths=None):
    q, k, v, do = (x[name].double() for name in ("q", "k", "v", "dout"))
    n, B, T, H, K = q.shape
    length = torch.full((n, B), T, device="cuda") if lengths is None else lengths.clamp(0, T)
    zero = torch.zeros(n, B, H, K, v.shape[-1], dtype=torch.float64, device="cuda")
    S = zero if x["state"] is None else x["state"].double()
    R = zero if x["dstate"] is None else x["dstate"].double()
    decay = torch.exp(x["log_decay"].double())[:, None, :, None, None]
    out, dq, dk, dv = torch.zeros_like(v), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for t in range(T):
        on = (t < length)[:, :, None, None]
        S = torch.where(on[..., None], decay * S + k[:, :, t, :, :, None] * v[:, :, t, :, None, :], S)
        out[:, :, t] = torch.where(on, scale * (q[:, :, t, :, :, None] * S).sum(-2), 0.0)
        dq[:, :, t] = torch.where(on, scale * (do[:, :, t, :, None, :] * S).sum(-1), 0.0)
    for t in range(T - 1, -1, -1):
        on = (t < length)[:, :, None, None]
        here = R + scale * q[:, :, t, :, :, None] * do[:, :, t, :, None, :]
        dk[:, :, t] = torch.where(on, (here * v[:, :, t, :, None, :]).sum(-1), 0.0)
        dv[:, :, t] = torch.where(on, (here * k[:, :, t, :, :, None]).sum(-2), 0.0)
        R = torch.where(on[..., None], decay * here, R)
    return {"out": out, "state": S, "dq": dq, "dk": dk, "dv": dv, "dstate": R}


def run(ops, x, scale, lengths=None):
    rest = {"scale": scale, "state": x["state"], "lengths": lengths}
    out, state = ops.linear_attention_forward(x["q"], x["k"], x["v"], x["log_decay"], **rest)
    dq, dk, dv, dstate = ops.linear_attention_backward(x["dout"], x["dstate"], x["q"], x["k"], x["v"], x["log_decay"], **rest)
    return {"out": out, "state": state, "dq": dq, "dk": dk, "dv": dv, "dstate": dstate}


def check(ops, x, scale=0.3, lengths=None):
    got = run(ops, x, scale, lengths)
    torch.cuda.synchronize()
    clean = x
    if lengths is not None:  # what the rows behind a sequence hold is not read
        on = (torch.arange(x["q"].shape[2], device="cuda") < lengths[:, :, None])[..., None, None]
        clean = {name: torch.where(on, t, 0.0) if name in ("q", "k", "v", "dout") else t for name, t in x.items()}
    want = definition(clean, scale, lengths)
    size = definition({name: t if t is None or name == "log_decay" else t.abs() for name, t in clean.items()}, abs(scale), lengths)
    dtype = x["q"].dtype
    T, K, W = x["q"].shape[2], x["q"].shape[-1], x["v"].shape[-1]
    sums = (6 * (K + W + 64) / 16 + T / 64 + 128 + 8) * 2.0 ** -23
    for name, t in got.items():
        assert t.shape == want[name].shape and t.dtype == (torch.float32 if "state" in name else dtype) and t.is_contiguous(), name
        half = dtype == torch.bfloat16
        term = sums + (2.0 ** -8 if half and "state" not in name else 2.0 ** -21)
        rounding = torch.finfo(t.dtype).eps / 2
        off = (t - want[name]).abs() - (term * size[name] + rounding * want[name].abs() + 2.0 ** -100)
        assert (off <= 0).all(), (name, float(off.max()))
        near = 5e-3 if half and "state" not in name else 5e-6
        assert (t - want[name]).norm() <= near * want[name].norm(), (name, float((t - want[name]).norm() / want[name].norm()))
    return got


SIZES = [(1, 1, 1, 1, 1, 1), (1, 1, 2, 1, 3, 5), (2, 3, 5, 2, 16, 16), (1, 2, 63, 3, 64, 64), (3, 1, 64, 2, 32, 128), (1, 1, 65, 1, 128, 128), (2, 2, 130, 3, 48, 40),
         (1, 3, 200, 2, 17, 33), (1, 1, 127, 2, 65, 127), (4, 2, 100, 1, 8, 100), (64, 1, 20, 2, 24, 10), (1, 2, 500, 3, 100, 72), (1, 5, 129, 7, 80, 64)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,B,T,H,K,W", SIZES)
def test_sizes(ops, dtype, n, B, T, H, K, W):
    check(ops, inputs(dtype, n, B, T, H, K, W, seed=T))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,B,T,H,K,W", [(1, 1, 1000, 2, 64, 64), (1, 1, 4111, 1, 128, 128), (2, 1, 3000, 3, 33, 65), (1, 1, 20000, 1, 16, 24)])
def test_long_sequences_of_few_heads(ops, dtype, n, B, T, H, K, W):
    """Sequences that are cut into segments, with and without first and last states, and heads that do not forget."""
    x = inputs(dtype, n, B, T, H, K, W, seed=1)
    check(ops, x)
    x["log_decay"][0, 0] = -1e-5
    x["state"], x["dstate"] = None, None
    check(ops, x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [70, 1000])
def test_lengths(ops, dtype, T):
    x = inputs(dtype, 2, 6, T, 2, 40, 24, seed=2)
    lengths = torch.tensor([[T, 0, 1, 64, T - 1, 33], [T // 2, 65, T + 5, -3, 63, 2]], device="cuda")
    for name in ("q", "k", "v", "dout"):
        x[name][(torch.arange(T, device="cuda") >= lengths[:, :, None])] = float("nan")
    got = check(ops, x, lengths=lengths)
    for name, first in (("state", "state"), ("dstate", "dstate")):
        assert torch.equal(got[name][0, 1], x[first][0, 1]) and torch.equal(got[name][1, 3], x[first][1, 3])
    x["state"], x["dstate"] = None, None
    got = check(ops, x, lengths=lengths)
    assert (got["state"][0, 1] == 0).all() and (got["dstate"][1, 3] == 0).all()


@pytest.mark.parametrize("K,W", [(33, 40), (40, 33), (85, 98), (1, 127), (120, 2)])
@pytest.mark.parametrize("T", [129, 192, 193, 700])
def test_columns_that_are_not_in_eights(ops, K, W, T):
    """bf16 heads of odd sizes in sequences of several lengths, as dense arrays, as parts of a projection's output, and at an odd address: whether
    copies are made of some, of all or of none of them, the rows behind a sequence are not read and those of results are zeros."""
    n, B, H = 2, 3, 5
    x = inputs("bf16", n, B, T, H, K, W, seed=T)
    lengths = torch.tensor([[T, 0, 1], [128, T - 1, 130]], device="cuda")
    for name in ("q", "k", "v", "dout"):
        x[name][(torch.arange(T, device="cuda") >= lengths[:, :, None])] = float("nan")
    check(ops, x, lengths=lengths)
    room = torch.full((n * B * T * H * (2 * K + W + 3) + 1,), float("nan"), dtype=torch.bfloat16, device="cuda")
    for shift in (0, 1):
        joint = room[shift:room.numel() - 1 + shift].view(n, B, T, H, 2 * K + W + 3)
        y = dict(x, q=joint[..., :K], k=joint[..., K:2 * K], v=joint[..., 2 * K:2 * K + W])
        for name in ("q", "k", "v"):
            y[name].copy_(x[name])
        check(ops, y, lengths=lengths)
    one = room[1:1 + x["v"].numel()].view_as(x["v"])
    one.copy_(x["v"])
    check(ops, dict(x, v=one, state=None, dstate=None), lengths=lengths)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_tokens_and_no_sequences(ops, dtype):
    x = inputs(dtype, 2, 3, 0, 2, 16, 8)
    got = run(ops, x, 1.0)
    assert got["out"].shape == (2, 3, 0, 2, 8) and torch.equal(got["state"], x["state"]) and torch.equal(got["dstate"], x["dstate"])
    x["state"], x["dstate"] = None, None
    got = run(ops, x, 1.0)
    assert (got["state"] == 0).all() and (got["dstate"] == 0).all()
    got = run(ops, inputs(dtype, 2, 0, 5, 2, 16, 8), 1.0)
    assert got["dq"].shape == (2, 0, 5, 2, 16) and got["state"].shape == (2, 0, 2, 16, 8)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decays_at_the_ends_of_their_range(ops, dtype):
    """A decay of zero keeps each token to itself, one of one forgets nothing; a positive log_decay or NaN spoils its own head alone."""
    x = inputs(dtype, 1, 2, 300, 4, 32, 32, seed=3)
    x["log_decay"][0] = torch.tensor([float("-inf"), 0.0, -200.0, -1e-30])
    check(ops, x)
    x["log_decay"][0] = torch.tensor([0.1, -0.1, float("nan"), -0.2])
    got = run(ops, x, 0.3)
    for name, t in got.items():
        t = t if "state" in name else t.transpose(2, 3)
        assert torch.isfinite(t[:, :, 1::2]).all() and torch.isnan(t[:, :, ::2]).any(), name
    assert torch.isnan(got["out"][:, :, :, ::2]).all() and torch.isnan(got["state"][:, :, ::2]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K,W,shift", [(64, 64, 0), (32, 48, 8), (64, 64, 2), (33, 31, 1)])
def test_strides_and_addresses(ops, dtype, K, W, shift):
    """Parts of one projection's output, axes in another order, addresses of every alignment: all hold to the definition.  fp32 results are those
    of dense copies; bf16 operands go through one kernel or another by how they lie, which round the same sums in other places (chunks of
    64 or of 128 tokens), so there the definition's bounds are all that both share."""
    n, B, T, H = 2, 3, 150, 2
    same = lambda a, b: dtype == "bf16" or all(torch.equal(a[name], b[name]) for name in b)  # noqa: E731
    x = inputs(dtype, n, B, T, H, K, W, seed=4)
    want = run(ops, x, 0.5)
    joint = torch.zeros(n, B, T, H, 2 * K + W + shift, dtype=TYPES[dtype], device="cuda")
    y = dict(x, q=joint[..., shift:shift + K], k=joint[..., shift + K:shift + 2 * K], v=joint[..., shift + 2 * K:])
    for name in ("q", "k", "v"):
        y[name].copy_(x[name])
    y["dout"] = x["dout"].permute(3, 1, 0, 2, 4).contiguous().permute(2, 1, 3, 0, 4)
    assert same(check(ops, y, 0.5), want)
    # broadcast inputs
    one = dict(x, k=x["k"][:, :, :, :1].expand(n, B, T, H, K), q=x["q"][:1].expand(n, B, T, H, K))
    dense = {name: None if t is None else t.contiguous() for name, t in one.items()}
    assert same(check(ops, one, 0.5), run(ops, dense, 0.5))
    spread = dict(x, v=x["v"][:, :, :1].expand(n, B, T, H, W), dout=x["dout"][:, :1].expand(n, B, T, H, W))
    check(ops, spread, 0.5)
    # a worker by itself
    single = {name: t[1] for name, t in x.items()}
    got = run(ops, single, 0.5)
    assert all(torch.equal(got[name], want[name][1]) for name in want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,B,H,K,W", [(1, 1, 1, 1, 1), (1, 8, 4, 64, 64), (2, 3, 2, 128, 128), (1, 5, 3, 17, 33), (3, 2, 2, 100, 127), (1, 2, 1, 128, 4), (1, 300, 5, 20, 12)])
def test_single_tokens(ops, dtype, n, B, H, K, W):
    """In fp32 throughout: a state is off by three roundings of its two terms, a result by those and a sum of K."""
    x = inputs(dtype, n, B, 1, H, K, W, seed=5)
    q, k, v = (x[name][:, :, 0] for name in "qkv")
    decay = torch.exp(x["log_decay"].double())[:, None, :, None, None]
    kv = k.double()[..., :, None] * v.double()[..., None, :]
    state = decay * x["state"] + kv
    size = decay * x["state"].abs() + kv.abs()
    want, out_size = 0.3 * (q.double()[..., None] * state).sum(-2), 0.3 * (q.double().abs()[..., None] * size).sum(-2)
    before, new = x["state"].clone(), torch.empty_like(x["state"])
    out = ops.linear_attention_step(q, k, v, x["log_decay"], x["state"], scale=0.3, new_state=new)
    assert torch.equal(before, x["state"])
    assert ((new - state).abs() <= 3 * 2.0 ** -24 * size).all()
    assert out.dtype == TYPES[dtype] and ((out - want).abs() <= (K + 8) * 2.0 ** -24 * out_size + torch.finfo(out.dtype).eps / 2 * want.abs()).all()
    again = ops.linear_attention_step(q, k, v, x["log_decay"], x["state"], scale=0.3)
    assert torch.equal(again, out) and torch.equal(x["state"], new)
    # strided, at any address
    joint = torch.cat([v, q, k, v[..., :1]], -1)[..., :-1]
    got = ops.linear_attention_step(joint[..., W:W + K], joint[..., W + K:], joint[..., :W], x["log_decay"], before, scale=0.3)
    assert torch.equal(got, out) and torch.equal(before, new)
    single = ops.linear_attention_step(q[0], k[0], v[0], x["log_decay"][0], x["state"][0], scale=0.3)
    assert torch.isfinite(single).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_steps_and_parts_go_on_where_a_sequence_ends(ops, dtype):
    """A prompt in one pass and the rest token by token, or in two parts, is the whole sequence: both sides hold to the definition."""
    x = inputs(dtype, 1, 2, 150, 3, 32, 48, seed=6)
    want = definition(x, 32 ** -0.5)
    out, state = ops.linear_attention_forward(*(x[name][:, :, :140] for name in "qkv"), x["log_decay"], state=x["state"])
    parts = [out]
    for t in range(140, 150):
        parts.append(ops.linear_attention_step(*(x[name][:, :, t] for name in "qkv"), x["log_decay"], state)[:, :, None])
    out = torch.cat(parts, 2)
    near = 5e-3 if dtype == "bf16" else 5e-6
    assert (out - want["out"]).norm() <= near * want["out"].norm()
    assert (state - want["state"]).norm() <= 5e-6 * want["state"].norm()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_through_autograd(ops, dtype):
    x = inputs(dtype, 2, 2, 90, 2, 24, 40, seed=7)
    lengths = torch.tensor([[90, 20], [64, 0]], device="cuda")
    want = run(ops, x, 0.5, lengths)
    leaves = {name: x[name].clone().requires_grad_() for name in ("q", "k", "v", "state")}
    out, state = ops.linear_attention(leaves["q"], leaves["k"], leaves["v"], x["log_decay"], scale=0.5, state=leaves["state"], lengths=lengths)
    torch.autograd.backward([out, state], [x["dout"], x["dstate"]])
    assert torch.equal(out, want["out"]) and torch.equal(state, want["state"])
    for name, grad in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("state", "dstate")):
        assert torch.equal(leaves[name].grad, want[grad]), name
    # one result used, the other not; the default scale
    for used in (0, 1):
        leaves = {name: x[name].clone().requires_grad_() for name in "qkv"}
        result = ops.linear_attention(leaves["q"], leaves["k"], leaves["v"], x["log_decay"])[used]
        result.sum().backward()
        y = dict(x, state=None, dout=torch.full_like(x["dout"], 1.0 - used), dstate=torch.full_like(x["dstate"], float(used)))
        got = run(ops, y, 24 ** -0.5)
        assert all(torch.equal(leaves[name].grad, got["d" + name]) for name in "qkv")


def test_gradients_of_differences(ops):
    """Each input enters linearly, so a change along a direction is the gradient's product with it, up to the fp32 roundings of both
    sides (their terms' sizes)."""
    x = inputs("f32", 1, 2, 140, 2, 20, 28, seed=8)
    got = run(ops, x, 0.4)

    def loss(y):
        r = run(ops, y, 0.4)
        return (r["out"].double() * x["dout"]).sum() + (r["state"].double() * x["dstate"]).sum()

    sizes = definition({name: t if name == "log_decay" else t.abs() for name, t in x.items()}, 0.4)
    total = float((sizes["out"] * x["dout"].abs()).sum() + (sizes["state"] * x["dstate"].abs()).sum())
    for name, grad in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("state", "dstate")):
        step = torch.randn_like(x[name])
        change = loss(dict(x, **{name: x[name] + step})) - loss(dict(x, **{name: x[name] - step}))
        assert abs(float(change / 2 - (got[grad].double() * step).sum())) <= 100 * 2.0 ** -23 * total, name


def test_infinities_and_nan_stay_in_their_chunk_and_what_follows(ops):
    x = inputs("f32", 2, 2, 200, 2, 16, 16, seed=9)
    clean = run(ops, x, 0.5)
    x["v"][1, 0, 130, 1, 3], x["k"][0, 1, 70, 0, 2] = float("nan"), float("inf")
    got = run(ops, x, 0.5)
    for name in ("out", "dq", "dk", "dv"):
        same = torch.ones_like(got[name], dtype=torch.bool)
        same[1, 0, :, 1], same[0, 1, :, 0] = False, False
        assert torch.equal(got[name][same], clean[name][same]), name
    assert torch.equal(got["out"][1, 0, :128, 1], clean["out"][1, 0, :128, 1]) and torch.isnan(got["out"][1, 0, 130:, 1, 3]).all()
    assert torch.equal(got["out"][0, 1, :64, 0], clean["out"][0, 1, :64, 0]) and not torch.isfinite(got["out"][0, 1, 70:, 0]).any()


def test_the_same_bits_every_time_in_graphs_and_on_other_streams(ops):
    x = inputs("bf16", 1, 2, 1500, 2, 64, 64, seed=10)
    held_state = x["state"].clone()

    def step():
        r = run(ops, x, 0.5)
        return list(r.values()) + [ops.linear_attention_step(x["q"][:, :, 0], x["k"][:, :, 0], x["v"][:, :, 0], x["log_decay"], held_state, new_state=torch.empty_like(held_state))]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in (11, 12):
        for name, t in inputs("bf16", 1, 2, 1500, 2, 64, 64, seed=seed).items():
            x[name].copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = step()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(held, again))


def test_offsets_past_32_bits(ops):
    """2^31 elements and more in every tensor.  Heads that forget at once: each result is its own token's."""
    T, H, D = 270_000, 64, 128
    x = torch.zeros(1, T, H, D, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(1, 3, H, D, device="cuda").bfloat16()
    x[:, -3:] = tail
    never = torch.full((H,), float("-inf"), device="cuda")
    out, state = ops.linear_attention_forward(x, x, x, never, scale=1.0)
    t = tail.double()
    want = t.square().sum(-1, keepdim=True) * t
    assert not out[:, :-3].any() and (out[:, -3:] - want).norm() <= 5e-3 * want.norm()
    last = t[:, -1, :, :, None] * t[:, -1, :, None, :]
    assert (state - last).norm() <= 5e-6 * last.norm()
    del out
    dq, dk, dv, first = ops.linear_attention_backward(x, None, x, x, x, never, scale=1.0)
    for grad in (dq, dk, dv):
        assert not grad[:, :-3].any() and (grad[:, -3:] - want).norm() <= 5e-3 * want.norm()
    assert not first.any()


def test_arguments_are_refused(ops):
    x = inputs("f32", 2, 3, 5, 2, 16, 8)
    q, k, v, ld, s, do = (x[name] for name in ("q", "k", "v", "log_decay", "state", "dout"))
    wide = torch.zeros(2, 3, 5, 2, 129, device="cuda")
    lengths = torch.ones(2, 3, dtype=torch.int64, device="cuda")
    f, b, t = ops.linear_attention_forward, ops.linear_attention_backward, ops.linear_attention_step
    q1, k1, v1 = q[:, :, 0], k[:, :, 0], v[:, :, 0]
    for call, match in ((lambda: f(q.cpu(), k, v, ld), "CUDA"), (lambda: f(q, k[:, :, :4], v, ld), "k must have shape"), (lambda: f(q, k, v[:, :, :4], ld), "v must have shape"),
                        (lambda: f(q, k.bfloat16(), v, ld), "type"), (lambda: f(q.half(), k.half(), v.half(), ld), "float32 or bfloat16"), (lambda: f(q[0, 0], k[0, 0], v[0, 0], ld), "q must be"),
                        (lambda: f(q, k, v, ld[0]), "log_decay must be"), (lambda: f(q, k, v, ld.double()), "log_decay must be"), (lambda: f(q, k, v[..., 0], ld), "v must have the axes"),
                        (lambda: f(q, k, v, ld, state=s[:1]), "state must be"), (lambda: f(q, k, v, ld, state=s.transpose(3, 4)), "state must be"),
                        (lambda: f(q, k, v, ld, state=s.bfloat16()), "state must be"), (lambda: f(q, k, v, ld, lengths=lengths.int()), "lengths must be"),
                        (lambda: f(q, k, v, ld, lengths=lengths[0]), "lengths must be"), (lambda: f(q, k, v, ld, scale=float("nan")), "scale"),
                        (lambda: f(wide, wide, v, ld), "128"), (lambda: f(q, k, wide, ld), "128"), (lambda: f(q[..., ::2], k[..., ::2], v, ld), "contiguous"),
                        (lambda: b(do[:, :, :4], None, q, k, v, ld), "dout must have shape"), (lambda: b(do, s[:1], q, k, v, ld), "dstate must be"),
                        (lambda: t(q1, k1, v1, ld, s[:1]), "state must be"), (lambda: t(q, k, v, ld, s), "must"), (lambda: t(q1, k1, v1, ld, s, new_state=s[..., :4]), "new_state must be"),
                        (lambda: t(q1, k1, v1, ld, torch.zeros(s.numel() + 4, device="cuda")[:s.numel()].view_as(s), new_state=s.flatten()[:0].view(0)), "new_state must be"),
                        (lambda: ops.linear_attention(q, k, v, ld.requires_grad_()), "no gradient")):
        with pytest.raises((ValueError, ops.RPSError), match=match):
            call()
    room = torch.zeros(s.numel() + 4, device="cuda")
    with pytest.raises(ValueError, match="overlaps"):
        t(q1, k1, v1, ld.detach(), room[:-4].view_as(s), new_state=room[4:].view_as(s))


def test_a_step_records_no_gradient(ops):
    """It is refused where one is wanted, and a gradient that needs the state from before it says so."""
    n, B, H, K = 1, 2, 2, 8
    q, k, v = (torch.randn(n, B, 3, H, K, device="cuda") for _ in "qkv")
    ld, state = torch.full((n, H), -0.1, device="cuda"), torch.randn(n, B, H, K, K, device="cuda")
    one = [t[:, :, 0] for t in (q, k, v)]
    for i in range(3):
        with pytest.raises(ValueError, match="no gradient"):
            ops.linear_attention_step(*[t.clone().requires_grad_() if i == j else t for j, t in enumerate(one)], ld, state)
    with pytest.raises(ValueError, match="no gradient"):
        ops.linear_attention_step(*one, ld, state.clone().requires_grad_())
    leaf = q.clone().requires_grad_()
    out, _ = ops.linear_attention(leaf, k, v, ld, state=state)
    other = torch.empty_like(state)
    ops.linear_attention_step(*one, ld, state, new_state=other)
    torch.autograd.grad(out.sum(), leaf, retain_graph=True)
    with torch.no_grad():
        ops.linear_attention_step(leaf[:, :, 0], *one[1:], ld, state)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(out.sum(), leaf)
    with torch.inference_mode():
        ops.linear_attention_step(*one, ld, state.clone())


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("T,K,W", [(100, 64, 64), (3000, 128, 128), (5000, 40, 72)])
def test_a_wait_that_runs_out_is_reported(ops, backward, T, K, W):
    """No copies are issued, so the kernel's waits for data give up after 200 ms; it ends by itself and the next check says so.  After that
    the same call works."""
    import ctypes

    lib = ops._library()
    x = inputs("bf16", 1, 2, T, 3, K, W, seed=13)
    want = run(ops, x, 0.5)
    ops.check()
    d = ops.rps_linear_attention_desc(dtype=1, n=1, heads=3, wait_limit_ms=200, withhold_copies=1, sequences=2, tokens=T, key_cols=K, value_cols=W, scale=0.5)
    d.q = d.k = ops.rps_axis_strides(0, T * 3 * K, 3 * K, K)
    d.v = d.dout = ops.rps_axis_strides(0, T * 3 * W, 3 * W, W)
    size = ctypes.c_size_t()
    assert lib.rps_linear_attention_workspace(ctypes.byref(d), int(backward), ctypes.byref(size)) == 0
    ws = torch.zeros(size.value + 256, dtype=torch.uint8, device="cuda")
    p = {name: t.data_ptr() for name, t in x.items()}
    out = [torch.empty_like(t) for t in want.values()]
    o = dict(zip(want, (t.data_ptr() for t in out)))
    stream = torch.cuda.current_stream().cuda_stream
    if backward:
        assert lib.rps_linear_attention_backward(ctypes.byref(d), p["dout"], p["dstate"], p["q"], p["k"], p["v"], p["log_decay"], None, p["state"], o["dq"], o["dk"],
                                                 o["dv"], o["dstate"], ws.data_ptr(), size.value, stream) == 0
    else:
        assert lib.rps_linear_attention_forward(ctypes.byref(d), p["q"], p["k"], p["v"], p["log_decay"], None, p["state"], o["out"], o["state"], ws.data_ptr(),
                                                size.value, stream) == 0
    with pytest.raises(ops.RPSError, match="gave up"):
        ops.check()
    ops.check()      # reported once
    got = run(ops, x, 0.5)
    ops.check()
    assert all(torch.equal(got[name], want[name]) for name in want)
