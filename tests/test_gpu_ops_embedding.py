"""Rows looked up by token, and the table's gradient, against their definitions in 64 bits.

Tolerances, from the number formats (half = half a step of the type, 2^-8 of bf16, 2^-24 of fp32, relative):
  lookup    scale as fp32 and one product of fp32, one rounding to the type
  gradient  scale as fp32 and the product with it 2 * 2^-24; a sum of m terms in fp32, in any tree, m * 2^-24 of the sum of their sizes; with
            accumulate one more addition; one rounding to the type"""
import pytest
import torch

pytestmark = pytest.mark.gpu

E32 = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    from paper_1810_07766_b200 import build, ops

    build.build()
    return ops


def half(dtype):
    return torch.finfo(dtype).eps / 2


def inputs(dtype, n, T, V, D, seed=0, ignored=0.2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    weight = torch.randn(n, V, D, generator=g, device="cuda").to(TYPES[dtype])
    tokens = (torch.rand(n, T, generator=g, device="cuda") ** 3 * V).long().clamp(0, V - 1)
    tokens[torch.rand(n, T, generator=g, device="cuda") < ignored] = -100
    dout = torch.randn(n, T, D, generator=g, device="cuda").to(TYPES[dtype])
    return tokens, weight, dout


def check_lookup(ops, tokens, weight, scale):
    out = ops.embedding_forward(tokens, weight, scale=scale)
    at = torch.arange(weight.shape[0], device="cuda")[:, None]
    want = weight[at, tokens.clamp(min=0)].double() * scale
    want[tokens == -100] = 0
    assert out.dtype == weight.dtype and out.shape == want.shape
    assert ((out - want).abs() <= (half(out.dtype) + 3 * E32) * want.abs()).all()


def check_gradient(ops, tokens, weight, dout, scale, accumulate, dweight=None):
    n, V, D = weight.shape
    want, size = torch.zeros(n, V, D, dtype=torch.float64, device="cuda"), torch.zeros(n, V, D, dtype=torch.float64, device="cuda")
    most = 1
    for w in range(n):
        keep = tokens[w] != -100
        want[w].index_add_(0, tokens[w, keep], dout[w, keep].double())
        size[w].index_add_(0, tokens[w, keep], dout[w, keep].double().abs())
        if keep.any():
            most = max(most, int(torch.bincount(tokens[w, keep]).max()))
    want, size = want * scale, size * abs(scale)
    there = None
    if accumulate:
        there = torch.randn(n, V, D, device="cuda").to(weight.dtype)
        dweight = there.clone() if dweight is None else dweight.copy_(there)
        want, size = want + there, size + there.abs()
    got = ops.embedding_backward(dout, tokens, V, scale=scale, dweight=dweight, accumulate=accumulate)
    assert got.dtype == weight.dtype and got.shape == want.shape
    bound = (most + 4) * E32 * size + half(got.dtype) * want.abs()
    assert ((got - want).abs() <= bound).all(), float(((got - want).abs() - bound).max())
    if accumulate:
        untouched = size == there.abs()
        assert torch.equal(got[untouched], there[untouched])
    assert torch.equal(got, ops.embedding_backward(dout, tokens, V, scale=scale, dweight=there if accumulate else None, accumulate=accumulate))
    return got


SIZES = [(1, 1, 1, 1), (1, 1, 7, 3), (2, 3, 5, 7), (3, 31, 40, 64), (1, 33, 1000, 65), (4, 100, 30, 129), (2, 1024, 257, 72), (1, 1025, 300, 256), (64, 17, 90, 20),
         (2, 4096, 3, 40), (1, 4097, 70000, 33), (3, 5000, 513, 100), (1, 16384, 2000, 24), (2, 16385, 1000, 33), (1, 70001, 131072, 16), (1, 300, 50, 2051),
         (1, 512, 400, 36), (2, 513, 400, 36), (1, 300_001, 5000, 8),
         (2, 8192, 700, 20), (1, 8193, 700, 20), (1, 32769, 70000, 12), (1, 131072, 3000, 8), (2, 131073, 3000, 8)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,T,V,D", SIZES)
def test_sizes(ops, dtype, n, T, V, D):
    tokens, weight, dout = inputs(dtype, n, T, V, D, seed=T)
    check_lookup(ops, tokens, weight, 1.7)
    check_gradient(ops, tokens, weight, dout, 1.7, False)
    check_gradient(ops, tokens, weight, dout, 0.3, True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [40, 3000, 20000])
def test_one_word_in_every_place(ops, dtype, T):
    """A run over all tiles, in the table's first and last row; and runs whose ends are those of tiles."""
    n, V, D = 3, 1 << 17, 40
    tokens, weight, dout = inputs(dtype, n, T, V, D, ignored=0.0)
    tokens[0], tokens[1], tokens[2] = 0, V - 1, torch.arange(T, device="cuda") // 16
    check_lookup(ops, tokens, weight, 1.0)
    check_gradient(ops, tokens, weight, dout, 1.0, False)
    check_gradient(ops, tokens.flip(1), weight, dout, 1.0, True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 130, 33])
def test_parameters_in_rows_of_a_larger_array(ops, dtype, D):
    """Tables that are views into the workers' rows, on addresses of every alignment; what lies around them is left as it was."""
    n, T, V = 3, 200, 50
    tokens, weight, dout = inputs(dtype, n, T, V, D)
    for shift in (0, 1, 2, 8):
        flat = torch.full((n, shift + V * D + 24), 7.0, device="cuda").to(TYPES[dtype])
        view = flat[:, shift:shift + V * D].view(n, V, D)
        view.copy_(weight)
        check_lookup(ops, tokens, view, 2.0)
        check_gradient(ops, tokens, weight, dout, 2.0, False, dweight=view)
        check_gradient(ops, tokens, weight, dout, 2.0, True, dweight=view)
        assert (flat[:, :shift] == 7).all() and (flat[:, shift + V * D:] == 7).all()
        wide = torch.full((n, V, D + shift), 7.0, device="cuda").to(TYPES[dtype])
        check_gradient(ops, tokens, weight, dout, 2.0, False, dweight=wide[..., :D])
        assert (wide[..., D:] == 7).all()
        check_lookup(ops, tokens, wide[..., :D].copy_(weight), 2.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ignored_tokens_and_tokens_that_name_no_row(ops, dtype):
    tokens, weight, dout = inputs(dtype, 2, 50, 20, 40)
    dout[tokens == -100] = float("nan")   # not read
    check_gradient(ops, tokens, weight, torch.where(tokens[..., None] == -100, 0.0, dout), 1.0, False)
    want = ops.embedding_backward(torch.where(tokens[..., None] == -100, 0.0, dout), tokens, 20)
    assert torch.equal(ops.embedding_backward(dout, tokens, 20), want)
    for bad in (20, -1, 1 << 40, -(1 << 40)):
        wrong = torch.where(tokens == -100, bad, tokens)
        out = ops.embedding_forward(wrong, weight)
        assert torch.isnan(out[tokens == -100]).all() and torch.isfinite(out[tokens != -100]).all()
        assert torch.equal(ops.embedding_backward(dout, wrong, 20), want)
    # another number stands for ignored tokens, one that would name a row too
    out = ops.embedding_forward(tokens.clamp(min=0), weight, ignore_index=0)
    assert (out[tokens <= 0] == 0).all()
    assert (ops.embedding_backward(dout.nan_to_num(), tokens.clamp(min=0), 20, ignore_index=0)[:, 0] == 0).all()
    none = torch.full_like(tokens, -100)
    assert (ops.embedding_forward(none, weight) == 0).all() and (ops.embedding_backward(dout, none, 20) == 0).all()
    there = weight.clone()
    assert torch.equal(ops.embedding_backward(dout, none, 20, dweight=there, accumulate=True), weight)
    empty = tokens[:, :0]
    assert ops.embedding_forward(empty, weight).shape == (2, 0, 40)
    assert (ops.embedding_backward(dout[:, :0], empty, 20, dweight=there) == 0).all()
    there.copy_(weight)
    assert torch.equal(ops.embedding_backward(dout[:, :0], empty, 20, dweight=there, accumulate=True), weight)


def test_infinities_and_nan_stay_in_their_rows(ops):
    tokens, weight, dout = inputs("f32", 1, 60, 10, 24, ignored=0.0)
    tokens[0, 5], tokens[0, 9] = 3, 4
    dout[0, 5, 2], dout[0, 9, 7] = float("inf"), float("nan")
    got = ops.embedding_backward(dout, tokens, 10)
    bad = ~torch.isfinite(got[0])
    assert bad.sum() == 2 and bad[3, 2] and bad[4, 7]
    weight[0, 3, 1] = float("-inf")
    out = ops.embedding_forward(tokens, weight)
    assert torch.isinf(out[0, :, 1]).sum() == (tokens == 3).sum()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_a_worker_axis_and_through_autograd(ops, dtype):
    tokens, weight, dout = inputs(dtype, 2, 70, 33, 48)
    leaf = weight.clone().requires_grad_()
    out = ops.embedding(tokens, leaf, scale=0.5)
    out.backward(dout.transpose(0, 1).contiguous().transpose(0, 1))
    assert torch.equal(out, ops.embedding_forward(tokens, weight, scale=0.5))
    assert torch.equal(leaf.grad, ops.embedding_backward(dout, tokens, 33, scale=0.5))
    assert torch.equal(out[1], ops.embedding_forward(tokens[1], weight[1], scale=0.5))
    assert torch.equal(leaf.grad[1], ops.embedding_backward(dout[1], tokens[1], 33, scale=0.5))
    # tokens that do not follow one another in memory, gradients of an expanded tensor
    spread = torch.stack([tokens, tokens], -1)[..., 0]
    assert torch.equal(ops.embedding_forward(spread, weight, scale=0.5), out)
    leaf = weight.clone().requires_grad_()
    ops.embedding(tokens, leaf).sum().backward()
    assert torch.equal(leaf.grad, ops.embedding_backward(torch.ones_like(dout), tokens, 33))


def test_gradient_of_differences(ops):
    """The loss changes along a direction of the table by the gradient's product with it (linear, so up to rounding: sums of 60 * 24 terms)."""
    tokens, weight, dout = inputs("f32", 2, 60, 10, 24)
    step = torch.randn_like(weight)
    change = (ops.embedding_forward(tokens, weight + step, scale=1.5).double() - ops.embedding_forward(tokens, weight, scale=1.5).double())
    grad = ops.embedding_backward(dout, tokens, 10, scale=1.5)
    a, b = (change * dout).sum(), (grad.double() * step).sum()
    assert abs(a - b) <= 2.0 ** -20 * (change.abs() * dout.abs()).sum()


def test_arguments_are_refused(ops):
    tokens, weight, dout = inputs("f32", 2, 10, 8, 16)
    for call, match in ((lambda: ops.embedding_forward(tokens.int(), weight), "int64"), (lambda: ops.embedding_forward(tokens[0], weight), "weight must be"),
                        (lambda: ops.embedding_forward(tokens, weight[:1]), "weight must have shape"), (lambda: ops.embedding_forward(tokens, weight.half()), "float32 or bfloat16"),
                        (lambda: ops.embedding_forward(tokens.cpu(), weight), "CUDA"), (lambda: ops.embedding_forward(tokens, weight.mT), "contiguous"),
                        (lambda: ops.embedding_backward(dout, tokens, 8, accumulate=True), "accumulate needs"),
                        (lambda: ops.embedding_backward(dout[:, :9], tokens, 8), "dout must have shape"),
                        (lambda: ops.embedding_backward(dout.transpose(0, 1).contiguous().transpose(0, 1), tokens, 8), "contiguous"),
                        (lambda: ops.embedding_backward(dout, tokens, 8, dweight=weight[:, :7]), "dweight must have shape"),
                        (lambda: ops.embedding_backward(dout, tokens, 8, dweight=weight.bfloat16()), "type"),
                        (lambda: ops.embedding_backward(dout, tokens, 8, dweight=weight[:1].expand(2, 8, 16)), "overlap"),
                        (lambda: ops.embedding_backward(dout, tokens, 0), "vocab"),
                        (lambda: ops.embedding_forward(tokens, weight, scale=float("inf")), "scale"),
                        (lambda: ops.embedding(tokens, weight, scale=torch.ones((), requires_grad=True)), "no gradient")):
        with pytest.raises((ValueError, ops.RPSError), match=match):
            call()


def test_calls_in_a_cuda_graph_and_on_another_stream(ops):
    tokens, weight, dout = inputs("bf16", 2, 3000, 500, 72)
    step = lambda: (ops.embedding_forward(tokens, weight), ops.embedding_backward(dout, tokens, 500))  # noqa: E731
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in (1, 2):
        a, b, c = inputs("bf16", 2, 3000, 500, 72, seed=seed)
        tokens.copy_(a), weight.copy_(b), dout.copy_(c)
        graph.replay()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = step()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(x, y) for x, y in zip(held, again))


def test_tables_past_32_bit_offsets(ops):
    """2^31 elements and more: the last rows are found and their gradients land there."""
    V, D = 300_000, 8192
    weight = torch.zeros(1, V, D, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(1, 3, D, device="cuda").bfloat16()
    weight[:, -3:] = tail
    tokens = torch.tensor([[V - 1, 0, V - 3, V - 2, V - 1]], device="cuda")
    assert torch.equal(ops.embedding_forward(tokens, weight), weight[:, tokens[0]])
    dout = torch.randn(1, 5, D, device="cuda").bfloat16()
    got = ops.embedding_backward(dout, tokens, V, dweight=weight)
    assert torch.equal(got[:, -3:], torch.stack([dout[:, 2], dout[:, 3], (dout[:, 0].float() + dout[:, 4].float()).bfloat16()], 1))
    assert torch.equal(got[:, 0], dout[:, 1]) and not got[:, 1:-3].any()
