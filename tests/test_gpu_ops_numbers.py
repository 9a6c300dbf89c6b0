"""Numbers at the ends of their ranges: logits and sums that are large or long, the parts that stand for fp32 values, infinities, and operands
with more pieces than 32 bits count."""
import pytest
import torch

from test_gpu_ops_loss import E32, ops  # noqa: F401

pytestmark = pytest.mark.gpu


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
