"""The step between two blocks, 8-bit activations and the weight gradient out of them, against their definitions in 64 bits.

Tolerances, from the number formats: e16 = 2^-8 (half a unit of bf16), e32 = 2^-23.  A row's statistics are sums of at most 16384 fp32
terms, added in a tree: relative error below 2^-18; an element is a handful of fp32 operations on terms whose sizes the test
adds up, so it is held to 2^-17 of that sum and one rounding to the result's type.  Sums over rows add (rows + 16) e32."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

E16, E32, ROW = 2.0 ** -8, 2.0 ** -23, 2.0 ** -17
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    from paper_1810_07766_b200 import build, ops

    build.build()
    return ops


def rounding(dtype):
    return E16 if dtype == "bf16" else E32


def norm_inputs(dtype, n, T, D, gates, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(TYPES[dtype])  # noqa: E731
    return {"x": r(n, T, D), "f": r(n, T, D) * 3, "gate": r(n, gates, D), "post": r(n, D), "pre": r(n, D), "dh": r(n, T, D), "dy": r(n, T, D)}


def forward_definition(s, scale):
    x, f, post, pre = (s[k].double() for k in ("x", "f", "post", "pre"))
    T, gates = x.shape[1], s["gate"].shape[1]
    gate = s["gate"].double().repeat_interleave(max(T // gates, 1), 1)[:, :T]
    post, pre = post[:, None], pre[:, None]
    rf = 1 / (f.square().mean(-1, keepdim=True) + EPS).sqrt()
    branch = scale * gate * f * rf * post
    h = x + branch
    rh = 1 / (h.square().mean(-1, keepdim=True) + EPS).sqrt()
    return h, x.abs() + branch.abs(), h * rh * pre, (x.abs() + branch.abs()) * rh * pre.abs(), rf[..., 0], rh[..., 0]


def backward_definition(s, f, h, rf, rh, scale, dh):
    """Gradients for the kept f, h, rf, rh, and the sums of the terms' sizes."""
    n, T, D = f.shape
    gates = s["gate"].shape[1]
    rows = max(T // gates, 1)
    f, h, rf, rh, dy, post, pre = (v.double() for v in (f, h, rf[..., None], rh[..., None], s["dy"], s["post"][:, None], s["pre"][:, None]))
    gate = s["gate"].double().repeat_interleave(rows, 1)[:, :T]
    dh = dh.double() if dh is not None else torch.zeros_like(dy)
    a = dy * pre
    dx = dh + rh * (a - h * rh ** 2 * (a * h).mean(-1, keepdim=True))
    sx = dh.abs() + rh * (a.abs() + h.abs() * rh ** 2 * (a * h).abs().mean(-1, keepdim=True))
    b, sb = scale * gate * dx * post, (scale * gate * post).abs() * sx
    df = rf * (b - f * rf ** 2 * (b * f).mean(-1, keepdim=True))
    sf = rf * (sb + f.abs() * rf ** 2 * (sb * f.abs()).mean(-1, keepdim=True))
    u = f * rf * post
    group = lambda v: v.view(n, gates, rows, D).sum(2)  # noqa: E731
    return {"dx": (dx, sx, 0), "df": (df, sf, 0), "dgate": (group(scale * u * dx), group((scale * u).abs() * sx), rows),
            "dpost": ((scale * gate * dx * f * rf).sum(1), ((scale * gate * f * rf).abs() * sx).sum(1), T),
            "dpre": ((dy * h * rh).sum(1), (dy * h * rh).abs().sum(1), T)}


def close(name, got, want, size, dtype, rows=0):
    bound = (ROW + (rows + 16) * E32) * size + rounding(dtype) * want.abs()
    bad = (got.double() - want).abs() - bound
    assert (bad <= 0).all(), (name, float(bad.max()))


def check_norm(ops, dtype, s, keep="values", scale=0.7, use_dh=True):
    h, y, kept = ops.gated_residual_norm_forward(s["x"], s["f"], s["gate"], s["post"], s["pre"], scale=scale, eps=EPS, keep=keep)
    wh, sh, wy, sy, rf, rh = forward_definition(s, scale)
    close("h", h, wh, sh, dtype)
    close("y", y, wy, sy, dtype)
    # h is x + branch: cancelled rows have a larger relative error in their statistics
    assert ((kept.r_f - rf).abs() <= ROW * rf).all()
    assert ((kept.r_h - rh).abs() <= ROW * rh * (1 + sh.square().mean(-1) * rh ** 2)).all()
    if keep == "int8":
        f, hh = ops.unpack_activation(kept.f), ops.unpack_activation(kept.h)
        for got, packed in ((s["f"], kept.f), (h, kept.h)):
            again = ops.pack_activation(got)
            assert torch.equal(again.codes, packed.codes) and torch.equal(again.scales, packed.scales)
        values = lambda p: p.codes[..., :p.columns].double() * p.scales.double().repeat_interleave(128, -1)[..., :p.columns]  # noqa: E731
        f, hh = values(kept.f), values(kept.h)
    else:
        f, hh = s["f"], h
    dh = s["dh"] if use_dh else None
    got = ops.gated_residual_norm_backward(dh, s["dy"], kept, s["gate"], s["post"], s["pre"], scale=scale)
    want = backward_definition(s, f, hh, kept.r_f, kept.r_h, scale, dh)
    for name, g in zip(("dx", "df", "dgate", "dpost", "dpre"), got):
        close(name, g, *want[name][:2], dtype, want[name][2])
    return (h, y) + got


NORM_SIZES = [(1, 1, 1, 1), (1, 1, 4096, 1), (1, 2, 3, 2), (2, 7, 129, 7), (3, 24, 1000, 1), (1, 50, 64, 5), (2, 33, 257, 3), (1, 600, 1024, 1),
              (1, 1200, 72, 600), (4, 12, 2048, 6), (64, 3, 40, 1), (1, 5, 8192, 5), (1, 3, 16384, 1), (2, 4, 16383, 2), (1, 2000, 5, 2000),
              (1, 1500, 520, 2), (1, 9, 5000, 3)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("keep", ["values", "int8"])
@pytest.mark.parametrize("n,T,D,gates", NORM_SIZES)
def test_norm_sizes(ops, dtype, keep, n, T, D, gates):
    check_norm(ops, dtype, norm_inputs(dtype, n, T, D, gates), keep=keep)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_parameters_out_of_a_replica_array(ops, dtype):
    n, T, D = 3, 10, 100
    s = norm_inputs(dtype, n, T, D, 1)
    flat = torch.full((n, 1001), float("nan"), dtype=TYPES[dtype], device="cuda")
    for k, at in (("post", 1), ("pre", 102), ("gate", 203)):
        v = flat[:, at:at + D].view(s[k].shape)
        v.copy_(s[k])
        s[k] = v
    check_norm(ops, dtype, s)
    # one parameter for all workers
    for k in ("post", "pre", "gate"):
        s[k] = s[k][:1].expand(s[k].shape)
    check_norm(ops, dtype, s, keep="int8")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_on_unaligned_activations(ops, dtype):
    n, T, D = 2, 6, 264
    s = norm_inputs(dtype, n, T, D, 2)
    for k in ("x", "f", "dh", "dy"):
        room = torch.empty(n * T * D + 1, dtype=TYPES[dtype], device="cuda")
        v = room[1:].view(n, T, D)
        v.copy_(s[k])
        s[k] = v
    check_norm(ops, dtype, s)
    check_norm(ops, dtype, s, use_dh=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("keep", ["values", "int8"])
def test_norm_of_zero_rows_and_no_tokens(ops, dtype, keep):
    s = norm_inputs(dtype, 2, 4, 300, 1)
    s["f"][0] = 0          # a block that answers nothing
    s["x"][0, 1] = 0       # and a residual of nothing: h is a row of zeros
    check_norm(ops, dtype, s, keep=keep)
    e = {k: (v[:, :0] if k in ("x", "f", "dh", "dy") else v) for k, v in s.items()}
    h, y, kept = ops.gated_residual_norm_forward(e["x"], e["f"], e["gate"], e["post"], e["pre"], keep=keep)
    assert h.shape == y.shape == (2, 0, 300)
    got = ops.gated_residual_norm_backward(e["dh"], e["dy"], kept, e["gate"], e["post"], e["pre"])
    assert got[0].shape == (2, 0, 300) and all((g == 0).all() for g in got[2:])


def test_norm_rows_with_nan_or_infinity_stay_alone(ops):
    s = norm_inputs("f32", 1, 6, 200, 6)
    s["f"][0, 2, 5] = float("inf")
    s["x"][0, 4, 1] = float("nan")
    h, y, kept = ops.gated_residual_norm_forward(s["x"], s["f"], s["gate"], s["post"], s["pre"])
    dx, df, dgate, _, _ = ops.gated_residual_norm_backward(s["dh"], s["dy"], kept, s["gate"], s["post"], s["pre"])
    fine = torch.tensor([0, 1, 3, 5], device="cuda")
    for t in (h, y, dx, df, dgate):
        assert torch.isfinite(t[0, fine]).all()
    assert torch.isnan(y[0, 4]).all() and not torch.isfinite(y[0, 2]).all()


def test_norm_gradients_against_differences(ops):
    """Central differences in fp32 of L = <h, a> + <y, b> along each gradient.  The step moves L by 2e-3 of the terms' size;
    fp32 errors of the difference are below 1e-6 of it and the third derivative's part is second order in the step."""
    s = norm_inputs("f32", 2, 12, 96, 3, seed=5)
    names = ("x", "f", "gate", "post", "pre")
    leaves = [s[k].clone().requires_grad_() for k in names]
    value = lambda v: [(t.double() * w.double()).sum() for t, w in zip(ops.gated_residual_norm(*v, scale=0.5, eps=EPS), (s["dh"], s["dy"]))]  # noqa: E731
    sum(value(leaves)).backward()
    for i, k in enumerate(names):
        g = leaves[i].grad
        step = g * (0.02 * float(s[k].norm() / g.norm()))
        at = [s[j] for j in names]
        ends = []
        for sign in (1, -1):
            moved = list(at)
            moved[i] = at[i] + sign * step
            ends.append(float(sum(value(moved))))
        want = float((g.double() * step.double()).sum())
        assert (ends[0] - ends[1]) / 2 == pytest.approx(want, rel=1e-2), k


def test_norm_autograd_without_one_of_the_gradients(ops):
    s = norm_inputs("bf16", 1, 8, 64, 1)
    names = ("x", "f", "gate", "post", "pre")
    for which in (0, 1):
        leaves = [s[k].clone().requires_grad_() for k in names]
        ops.gated_residual_norm(*leaves, keep="int8")[which].float().sum().backward()
        h, y, kept = ops.gated_residual_norm_forward(*(s[k] for k in names), keep="int8")
        one, zero = torch.ones_like(h), torch.zeros_like(h)
        want = ops.gated_residual_norm_backward(one if which == 0 else None, zero if which == 0 else one, kept, s["gate"], s["post"], s["pre"])
        for a, b in zip(leaves, want):
            assert torch.equal(a.grad, b)


def test_norm_refusals(ops):
    s = norm_inputs("f32", 2, 6, 40, 3)
    a = [s[k] for k in ("x", "f", "gate", "post", "pre")]
    for i, bad in ((0, s["x"].half()), (0, s["x"].transpose(1, 2)), (1, s["f"].bfloat16()), (1, s["f"][:, :3]), (2, s["gate"][:, :, :3]), (3, s["post"][:1]),
                   (4, s["pre"].cpu()), (2, s["gate"][0]), (3, s["post"].repeat(1, 2)[:, ::2])):
        b = list(a)
        b[i] = bad
        with pytest.raises(ValueError):
            ops.gated_residual_norm_forward(*b)
    with pytest.raises(ValueError):
        ops.gated_residual_norm_forward(*a, keep="int4")
    with pytest.raises(ops.RPSError):   # 4 does not divide 6
        ops.gated_residual_norm_forward(a[0], a[1], torch.ones(2, 4, 40, device="cuda"), a[3], a[4])
    wide = torch.ones(1, 1, ops.MAX_NORM_COLS + 1, device="cuda")
    with pytest.raises(ops.RPSError):
        ops.gated_residual_norm_forward(wide, wide, wide, wide[0], wide[0])


# ------------------------------------------------------------------------------------------------------------- 8 bits
def pack_definition(x):
    """Codes and scales in float32, one operation at a time."""
    x = x.float().cpu().numpy()
    rows, cols = x.shape
    groups = -(-cols // 128)
    v = np.zeros((rows, groups * 128), np.float32)
    v[:, :cols] = x
    v = v.reshape(rows, groups, 128)
    with np.errstate(all="ignore"):
        top = np.abs(v).max(-1)
        bad = ~np.isfinite(v).all(-1)
        zero = bad | (top < np.float32(2.0 ** -100))
        factor = np.where(zero, np.float32(0), np.float32(127) / top).astype(np.float32)
        codes = np.where(zero[..., None], 0, np.rint(v * factor[..., None]))
    scale = np.where(bad, np.float32("nan"), np.where(zero, np.float32(0), top * (np.float32(1) / np.float32(127)))).astype(np.float32)
    return codes.reshape(rows, -1)[:, :cols].astype(np.int8), scale


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 128), (4, 129), (64, 1024), (17, 1000), (2, 40000), (3000, 33), (70, 4095)])
def test_pack_is_exact(ops, dtype, rows, cols):
    g = torch.Generator(device="cuda").manual_seed(rows * 1000 + cols)
    x = (torch.randn(rows, cols, generator=g, device="cuda") * torch.exp(3 * torch.randn(rows, 1, generator=g, device="cuda"))).to(TYPES[dtype])
    x[0] = 0
    x[-1, 0] = float("inf")
    if rows > 2:
        x[1, -1] = float("nan")
        x[2] = 1e-35
    p = ops.pack_activation(x)
    codes, scales = pack_definition(x)
    got = p.codes.cpu().numpy()
    assert np.array_equal(got[:, :cols], codes) and not got[:, cols:].any()
    assert np.array_equal(p.scales.cpu().numpy(), scales, equal_nan=True)
    back = ops.unpack_activation(p)
    want = torch.from_numpy(codes.astype(np.float32) * np.repeat(scales, 128, 1)[:, :cols]).cuda().to(TYPES[dtype])
    assert back.dtype == x.dtype and torch.equal(back.nan_to_num(7.0), want.nan_to_num(7.0))
    fine = torch.from_numpy(np.isfinite(np.repeat(scales, 128, 1)[:, :cols])).cuda()
    half = torch.from_numpy(np.repeat(scales, 128, 1)[:, :cols]).cuda().nan_to_num(0) * 0.5
    assert ((back.float() - x.float()).abs()[fine] <= (half * 1.001 + 2.0 ** -100 + (E16 * x.float().abs() if dtype == "bf16" else 0))[fine]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pack_of_strided_rows_more_axes_and_nothing(ops, dtype):
    x = torch.randn(20, 301, device="cuda").to(TYPES[dtype])
    a, b = ops.pack_activation(x[:, 1:300]), ops.pack_activation(x[:, 1:300].contiguous())
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    c = ops.pack_activation(x.view(4, 5, 301))
    assert c.codes.shape == (4, 5, 304) and c.scales.shape == (4, 5, 3) and ops.unpack_activation(c).shape == (4, 5, 301)
    empty = ops.pack_activation(x[:0])
    assert ops.unpack_activation(empty).shape == (0, 301)
    with pytest.raises(ValueError):
        ops.pack_activation(x.t())
    with pytest.raises(ValueError):
        ops.pack_activation(x.double())
    with pytest.raises(ValueError):
        ops.unpack_activation(a._replace(columns=400))
    with pytest.raises(ValueError):
        ops.unpack_activation(a._replace(scales=a.scales.double()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,T,O,D", [(1, 1, 1, 1), (2, 3, 5, 7), (1, 64, 64, 64), (3, 100, 130, 70), (8, 200, 300, 1001), (1, 1000, 257, 129),
                                     (1, 0, 20, 30), (1, 513, 264, 520), (64, 9, 16, 24)])
def test_packed_weight_grad(ops, dtype, n, T, O, D):
    g = torch.Generator(device="cuda").manual_seed(T)
    dy = torch.randn(n, T, O, generator=g, device="cuda").to(TYPES[dtype])
    x = (torch.randn(n, T, D, generator=g, device="cuda") * 3).to(TYPES[dtype])
    p = ops.pack_activation(x)
    kept = p.codes[..., :D].double() * p.scales.double().repeat_interleave(128, -1)[..., :D]
    want = dy.double().mT @ kept
    size = dy.double().abs().mT @ kept.abs()
    term = (E16 if dtype == "bf16" else 0.0) + (6 * T + 16) * E32
    got = ops.packed_weight_grad(dy, p)
    assert got.shape == (n, O, D) and got.dtype == dy.dtype
    assert ((got - want).abs() <= term * size + rounding(dtype) * want.abs()).all()
    assert (got - want).norm() <= (5e-3 if dtype == "bf16" else 1e-5) * want.norm() + 1e-300
    # a strided dy and a strided gradient
    wide = torch.full((n, T, O + 3), float("nan"), dtype=dy.dtype, device="cuda")
    wide[:, :, 1:O + 1] = dy
    out = torch.full((n, O, D + 1), 7.0, dtype=dy.dtype, device="cuda")
    ops.packed_weight_grad(wide[:, :, 1:O + 1], p, dweight=out[:, :, :D])
    assert torch.equal(out[:, :, :D], got) and (out[:, :, D:] == 7).all()


def test_linear_8bit(ops):
    x = torch.randn(2, 40, 96, device="cuda", dtype=torch.bfloat16).requires_grad_()
    w = (torch.randn(2, 72, 96, device="cuda") / 10).bfloat16().requires_grad_()
    y = ops.linear_8bit(x, w)
    dy = torch.randn_like(y)
    y.backward(dy)
    assert torch.equal(y, x.detach() @ w.detach().mT) and torch.equal(x.grad, dy @ w.detach())
    assert torch.equal(w.grad, ops.packed_weight_grad(dy, ops.pack_activation(x.detach())))
    # 8 bits: an element of x is off by at most 1/254 of its group's largest
    full = dy.double().mT @ x.detach().double()
    assert (w.grad - full).norm() <= 2e-2 * full.norm()
    with pytest.raises(ValueError):
        ops.packed_weight_grad(dy.float(), ops.pack_activation(x.detach()))
    with pytest.raises(ValueError):
        ops.packed_weight_grad(dy[:, :3], ops.pack_activation(x.detach()))
    with pytest.raises(ValueError):
        ops.linear_8bit(x, w[0])
