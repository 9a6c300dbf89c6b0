"""Numbers at the ends of their ranges: logits and sums that are large or long, the parts that stand for fp32 values, infinities, and operands
with more pieces than 32 bits count."""
import pytest
import torch

from test_gpu_ops_loss import E32, TYPES, check, inputs, ops  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 3, 40, 300])
@pytest.mark.parametrize("spread", [1e6, 1e10, 1e15])
def test_logits_of_any_size(ops, dtype, T, spread):  # noqa: F811
    """Where the largest logit is beyond 2^30, a unit of its last place is beyond the exponent's range: differences have to be formed
    before anything is scaled.  (All but one of a row's probabilities are zero, so the gradients are exact.)"""
    h, w, y = inputs(dtype, 2, T, 500, 48, seed=T, spread=spread)
    loss, lse, dh, dw = check(ops, dtype, h, w, y)
    assert torch.isfinite(loss).all() and torch.isfinite(dh).all() and torch.isfinite(dw).all()


def test_sums_over_many_tokens_are_not_cut_off(ops):  # noqa: F811
    """The tensor cores cut a sum off after each 16 terms.  2^19 tokens are 32768 such steps, which of a sum of terms of one sign take 3.2e-3 in one
    run; in runs of a few thousand steps it has to be 2.4e-4 at most, far below the rounding of a bf16 result (2e-3).  That rounding averages out
    here: the results' sizes are spread over a factor of four."""
    T, O, D = 1 << 19, 2304, 2304
    g = torch.Generator(device="cuda").manual_seed(1)
    dy = torch.empty(T, O, dtype=torch.bfloat16, device="cuda")
    codes = torch.empty(T, D, dtype=torch.int8, device="cuda")
    scales = torch.full((T, D // 128), 2.0 ** -7, device="cuda")
    up = torch.linspace(1, 2, O, device="cuda")
    want = torch.zeros(O, D, dtype=torch.float64, device="cuda")
    for t in range(0, T, 1 << 15):
        part = slice(t, t + (1 << 15))
        dy[part] = (torch.rand(1 << 15, O, generator=g, device="cuda") * 0.5 + 0.5) * up
        codes[part] = ((torch.rand(1 << 15, D, generator=g, device="cuda") * 30 + 30) * up).to(torch.int8)
        want += dy[part].double().T @ (codes[part].double() * 2.0 ** -7)
    got = ops.packed_weight_grad(dy, ops.PackedActivation(codes, scales, D, torch.bfloat16))
    off = got.double() / want - 1
    assert abs(float(off.mean())) <= 2.4e-4, float(off.mean())
    assert float(off.abs().max()) <= 2.0 ** -8 + 5e-4


def test_long_sums_of_odd_widths(ops):  # noqa: F811
    """Sums of more steps than one run holds, into rows that are not 16-byte aligned and past their last column."""
    T, O, D = 66000, 2303, 2311
    g = torch.Generator(device="cuda").manual_seed(6)
    dy = torch.randn(1, T, O, generator=g, device="cuda").bfloat16()
    p = ops.pack_activation(torch.randn(1, T, D, generator=g, device="cuda").bfloat16())
    x = ops.unpack_activation(p).double()   # as the product takes them: rounded to bf16
    out = torch.full((1, O, D + 1), 7.0, dtype=torch.bfloat16, device="cuda")
    ops.packed_weight_grad(dy, p, dweight=out[:, :, :D])
    want, size = dy[0].double().T @ x[0], dy[0].double().abs().T @ x[0].abs()
    assert (out[:, :, D] == 7).all()
    assert ((out[0, :, :D] - want).abs() <= 4096 * E32 * size + 2.0 ** -8 * want.abs()).all()
    assert (out[0, :, :D] - want).norm() <= 2.0 ** -8 * want.norm()


@pytest.mark.parametrize("T,V,D", [(2048, 70000, 2560), (5, 40, 70000)])  # dhidden sums over the words, logits over the columns
def test_long_sums_of_the_loss(ops, T, V, D):  # noqa: F811
    check(ops, "bf16", *inputs("bf16", 1, T, V, D, seed=7))


def test_fp32_products_keep_fp32_accuracy(ops):  # noqa: F811
    """A single token, so that each result is one product.  With three parts that are each rounded to nearest the six products made
    leave out at most 2^-24 of it; the last of their sums may be cut off by a unit, 2^-23."""
    g = torch.Generator(device="cuda").manual_seed(2)
    dy, x = torch.randn(1, 1, 2000, generator=g, device="cuda"), torch.randn(1, 1, 1920, generator=g, device="cuda")
    # every value of a group has a different exponent and all 24 bits
    p = ops.PackedActivation(torch.randint(1, 128, (1, 1, 1920), generator=g, device="cuda").to(torch.int8), x.abs()[..., :15].contiguous(), 1920, torch.float32)
    kept = ops.unpack_activation(p).double()
    got, want = ops.packed_weight_grad(dy, p).double(), dy.double().mT @ kept
    assert float((got / want - 1).abs().max()) <= 2.0 ** -22


@pytest.mark.parametrize("size,scale", [(3.4028e38, 1e-30), (3.3961e38, 2.0 ** -7), (1e30, 1e-30), (2.0 ** -108, 1.0)])
def test_fp32_products_of_the_largest_and_smallest_values(ops, size, scale):  # noqa: F811
    """Values that round to infinity as bf16, and values whose last part is the smallest that bf16 has: the bound of the test before."""
    dy = torch.full((1, 1, 64), size, device="cuda") * torch.linspace(0.9999, 1, 64, device="cuda")
    p = ops.PackedActivation((torch.arange(64, device="cuda") - 32).to(torch.int8)[None, None], torch.full((1, 1, 1), scale, device="cuda"), 64, torch.float32)
    got, want = ops.packed_weight_grad(dy, p).double(), dy.double().mT @ ops.unpack_activation(p).double()
    fits = want.abs() < 3.4e38
    assert fits[..., 31].all() and ((got - want).abs()[fits] <= 2.0 ** -22 * want.abs()[fits]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [3, 200])
def test_infinities_go_through_products(ops, dtype, T):  # noqa: F811
    """An infinity times a number is an infinity of the product's sign, times zero it is NaN; nothing else is touched."""
    O, D = 40, 260
    g = torch.Generator(device="cuda").manual_seed(3)
    dy = torch.randn(1, T, O, generator=g, device="cuda").to(TYPES[dtype])
    p = ops.pack_activation(torch.randn(1, T, D, generator=g, device="cuda").to(TYPES[dtype]))
    dy[0, 1, 3], dy[0, T - 1, 7], dy[0, 0, 9] = float("inf"), float("-inf"), float("nan")
    kept = ops.unpack_activation(p)
    want, got = dy.double().mT @ kept.double(), ops.packed_weight_grad(dy, p)
    rows = torch.ones(O, dtype=torch.bool)
    rows[[3, 7, 9]] = False
    assert torch.isfinite(got[0, rows.cuda()]).all()
    assert torch.isinf(want[0, 3]).any() and torch.isnan(want[0, 3]).sum() <= D // 4
    for o in (3, 7, 9):
        assert torch.equal(got[0, o].double().nan_to_num(nan=5.0), want[0, o].nan_to_num(nan=5.0)), o


def test_operands_of_more_than_2_to_the_32_pieces(ops):  # noqa: F811
    """A dy of 64 GiB and more whose rows have to be laid out anew: its last tokens count like its first."""
    T, O, D = 4_191_000, 8199, 16   # 1025 pieces of 16 bytes to a laid-out row
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("this test needs 150 GiB of device memory")
    dy = torch.zeros(T, O, dtype=torch.bfloat16, device="cuda")
    codes, scales = torch.zeros(T, D, dtype=torch.int8, device="cuda"), torch.ones(T, 1, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(4)
    tokens = torch.tensor([0, 5, 1000, T // 3, T // 2, T - 7, T - 1], device="cuda")
    dy[tokens] = torch.randn(7, O, generator=g, device="cuda").bfloat16()
    codes[tokens] = torch.randint(-127, 128, (7, D), generator=g, device="cuda").to(torch.int8)
    got = ops.packed_weight_grad(dy, ops.PackedActivation(codes, scales, D, torch.bfloat16))
    want = dy[tokens].double().T @ codes[tokens].double()
    size = dy[tokens].double().abs().T @ codes[tokens].double().abs()
    del dy
    torch.cuda.empty_cache()
    assert ((got - want).abs() <= 7 * E32 * size + 2.0 ** -8 * want.abs()).all()
