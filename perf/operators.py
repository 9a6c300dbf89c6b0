"""What the training operators are measured on: cases, inputs, a plain form of each operator in elementary torch operations,
the calls of the package that compute the same, and a definition in 64 bits to hold both against.

The package simulates ``n`` workers on one GPU, so every operator has a leading worker axis.  Three operators:

* ``loss``: softmax cross entropy of ``hidden @ weight.T`` over a large vocabulary, with its gradient;
* ``norm``: the step between two blocks of a network: norm after the block, gate, residual scale, residual sum, norm before
  the next block; forward alone, or forward and backward, the backward out of the kept values or out of 8-bit copies;
* ``pack``: activations kept in 8 bits with a scale for each 128 columns, there and back, and ``wgrad``: the weight gradient of
  a linear layer out of an input kept so.
"""
import math

import torch

own = False

IGNORE = -100
GROUP = 128
EPS = 1e-6
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # four workers with a small tagger's vocabulary and one short batch each: every call is launch latency
        {"name": "loss 4x32x1000 bf16", "op": "loss", "train": True, "dtype": "bf16", "n": 4, "T": 32, "V": 1000, "D": 256, "ignored": 0.0},
        # eight workers' training step on full-precision replicas, sizes that no tile divides; a quarter of the tokens is padding
        {"name": "loss 8x500x10001 f32", "op": "loss", "train": True, "dtype": "f32", "n": 8, "T": 500, "V": 10001, "D": 650, "ignored": 0.25},
        # evaluation: the loss of each token, no gradient, a vocabulary that no tile divides
        {"name": "loss eval 2048x50001 bf16", "op": "loss", "train": False, "dtype": "bf16", "n": 1, "T": 2048, "V": 50001, "D": 1024, "ignored": 0.0},
        # the largest: a long batch over a large vocabulary, prompts masked out of the loss
        {"name": "loss 4096x131072 bf16", "op": "loss", "train": True, "dtype": "bf16", "n": 1, "T": 4096, "V": 131072, "D": 2048, "ignored": 0.1},
        # a single token going forward: latency
        {"name": "norm 1x4096 bf16 forward", "op": "norm", "train": False, "dtype": "bf16", "n": 1, "T": 1, "D": 4096, "gates": 1, "keep": "values"},
        # eight workers in full precision, a learned gate for each channel
        {"name": "norm 8x256x1000 f32", "op": "norm", "train": True, "dtype": "f32", "n": 8, "T": 256, "D": 1000, "gates": 1, "keep": "values"},
        # a long batch, one gate value for each token and channel
        {"name": "norm 16384x4096 bf16", "op": "norm", "train": True, "dtype": "bf16", "n": 1, "T": 16384, "D": 4096, "gates": 16384, "keep": "values"},
        # four workers, a gate row for each of 8 sequences, the block's tensors kept in 8 bits for the backward pass
        {"name": "norm 4x2048x2048 bf16 8-bit", "op": "norm", "train": True, "dtype": "bf16", "n": 4, "T": 2048, "D": 2048, "gates": 8, "keep": "int8"},
        # a short batch's activations packed and read back
        {"name": "pack 64x1024 bf16", "op": "pack", "dtype": "bf16", "n": 1, "T": 64, "D": 1024},
        # a large set of activations in full precision, a width that is no multiple of the group
        {"name": "pack 4x8192x5000 f32", "op": "pack", "dtype": "f32", "n": 4, "T": 8192, "D": 5000},
        # eight workers' small full-precision layers, widths that no tile divides: weight gradient out of the packed input
        {"name": "wgrad 8x200x300x1001 f32", "op": "wgrad", "dtype": "f32", "n": 8, "T": 200, "V": 300, "D": 1001},
        # the same of one wide layer
        {"name": "wgrad 8192x8192x2048 bf16", "op": "wgrad", "dtype": "bf16", "n": 1, "T": 8192, "V": 8192, "D": 2048},
    ]


def _log_uniform(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    largest = max(work(c)["flops"] for c in listed())
    op = rng.choice(["loss", "loss", "norm", "norm", "pack", "wgrad"])
    while True:
        dtype = rng.choice(["bf16", "f32"])
        n = rng.choice([1, 1, 2, 3, 4, 8])
        if op == "loss":
            c = {"op": op, "train": rng.random() < 0.7, "dtype": dtype, "n": n, "T": _log_uniform(rng, 1, 8192),
                 "V": _log_uniform(rng, 100, 131072), "D": _log_uniform(rng, 64, 4096), "ignored": rng.choice([0.0, 0.1, 0.5])}
            if dtype == "f32" and work(c)["flops"] > largest / 8:
                continue
        elif op == "norm":
            seq = _log_uniform(rng, 1, 2048)
            seqs = _log_uniform(rng, 1, 16)
            train = rng.random() < 0.75
            c = {"op": op, "train": train, "dtype": dtype, "n": n, "T": seq * seqs, "D": _log_uniform(rng, 64, 8192),
                 "gates": rng.choice([1, seqs, seq * seqs]), "keep": "int8" if train and dtype == "bf16" and rng.random() < 0.4 else "values"}
        elif op == "pack":
            c = {"op": op, "dtype": dtype, "n": n, "T": _log_uniform(rng, 1, 16384), "D": _log_uniform(rng, 64, 8192)}
        else:
            c = {"op": op, "dtype": dtype, "n": n, "T": _log_uniform(rng, 1, 16384), "V": _log_uniform(rng, 64, 8192), "D": _log_uniform(rng, 64, 8192)}
        if c["n"] * c["T"] * c["D"] > 200_000_000:
            continue
        if op == "loss" and c["n"] * c["T"] * c["V"] > 4096 * 131072 or "V" in c and c["n"] * c["V"] * c["D"] > 300_000_000:
            continue
        if work(c)["flops"] <= (largest if op == "loss" else largest / 8):
            return c


# --------------------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype = _TYPES[case["dtype"]]
    n, T, D = case["n"], case["T"], case["D"]

    def normal(*shape, scale=1.0, offset=0.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale + offset).to(dtype)

    s = {"case": case}
    if case["op"] == "loss":
        V = case["V"]
        # normed activations and a head whose logits spread by about 2; frequent words have small numbers
        s["hidden"] = normal(n, T, D)
        s["weight"] = normal(n, V, D, scale=2.0 / math.sqrt(D))
        u = torch.rand(n, T, generator=g, device="cuda", dtype=torch.float64)
        y = (torch.exp(u * math.log(V + 1)) - 1).long().clamp(0, V - 1)
        # as many ignored tokens in every worker as the case says, at random places
        count = int(case["ignored"] * T)
        if count:
            place = torch.rand(n, T, generator=g, device="cuda").argsort(dim=1)[:, :count]
            y.scatter_(1, place, IGNORE)
        s["targets"] = y
        s["dloss"] = torch.rand(n, generator=g, device="cuda") + 0.5 if case["train"] else None
        return s
    if case["op"] == "norm":
        s["x"] = normal(n, T, D)
        # a block's output: some channels are far larger than the rest
        s["f"] = (torch.randn(n, T, D, generator=g, device="cuda") * _channels(n, D, g)).to(dtype)
        s["gate"] = normal(n, case["gates"], D, scale=0.3, offset=0.5)
        s["post"] = normal(n, D, scale=0.1, offset=1.0)
        s["pre"] = normal(n, D, scale=0.1, offset=1.0)
        s["scale"] = 0.7
        s["dh"], s["dy"] = (normal(n, T, D), normal(n, T, D)) if case["train"] else (None, None)
        return s
    x = (torch.randn(n, T, D, generator=g, device="cuda") * _channels(n, D, g)).to(dtype)
    if case["op"] == "pack":
        s["x"] = x
        return s
    # what the forward pass kept: codes with rows padded to 16 bytes, and a scale for each 128 columns
    codes, scales = _quantise(x)
    s["codes"] = torch.zeros(n, T, -(-D // 16) * 16, dtype=torch.int8, device="cuda")
    s["codes"][:, :, :D] = codes.to(torch.int8)
    s["scales"] = scales
    s["dy"] = normal(n, T, case["V"])
    return s


def _channels(n, D, g):
    """Spread of each channel: about one in fifty is twenty times the others."""
    return 1.0 + 19.0 * (torch.rand(n, 1, D, generator=g, device="cuda") < 0.02)


# ---------------------------------------------------------------------------------------------------------- plain forms
def _quantise(x):
    """Whole codes as float32 [n, T, D] and the float32 scales [n, T, groups]."""
    n, T, D = x.shape
    groups = -(-D // GROUP)
    v = torch.nn.functional.pad(x.float(), (0, groups * GROUP - D)).view(n, T, groups, GROUP)
    top = v.abs().amax(-1)
    codes = torch.round(v * torch.where(top > 0, torch.full_like(top, 127.0) / top, 0.0)[..., None])
    return codes.view(n, T, groups * GROUP)[:, :, :D], top * (1.0 / 127.0)


def _dequantise(codes, scales):
    D = codes.shape[-1]
    return codes.float() * scales.repeat_interleave(GROUP, dim=-1)[:, :, :D]


def _loss_plain(s):
    case, dtype, y = s["case"], s["hidden"].dtype, s["targets"]
    h, w = s["hidden"].float(), s["weight"].float()
    valid = y != IGNORE
    at = y.clamp(min=0)[..., None]
    logits = torch.bmm(h, w.transpose(1, 2))
    top = logits.amax(-1, keepdim=True)
    hit = logits.gather(-1, at)
    e = logits.sub_(top).exp_()
    z = e.sum(-1, keepdim=True)
    each = torch.where(valid, (top + z.log() - hit).squeeze(-1), 0.0)
    if not case["train"]:
        return {"loss": each, "lse": torch.where(valid, (top + z.log()).squeeze(-1), 0.0)}
    count = valid.sum(-1).clamp(min=1).float()
    c = torch.where(valid, (s["dloss"] / count)[:, None], 0.0)[..., None]
    dl = e.mul_(c / z)
    dl.scatter_add_(-1, at, -c)
    return {"loss": each.sum(-1) / count, "dhidden": torch.bmm(dl, w).to(dtype), "dweight": torch.bmm(dl.transpose(1, 2), h).to(dtype)}


def _norm_plain(s):
    case, dtype = s["case"], s["x"].dtype
    n, T, D = s["x"].shape
    x, f = s["x"].float(), s["f"].float()
    post, pre = s["post"].float()[:, None], s["pre"].float()[:, None]
    rows = T // case["gates"]
    gate = s["gate"].float().repeat_interleave(rows, dim=1)
    r_f = torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS)
    u = f * r_f * post
    h = x + s["scale"] * gate * u
    r_h = torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS)
    out = {"h": h.to(dtype), "y": (h * r_h * pre).to(dtype)}
    if not case["train"]:
        return out
    dh, dy = s["dh"].float(), s["dy"].float()
    if case["keep"] == "int8":
        # what the backward pass reads are the 8-bit copies of f and of h in the tensors' type
        f, h = _dequantise(*_quantise(s["f"])), _dequantise(*_quantise(out["h"]))
        u = f * r_f * post
    a = dy * pre
    dh = dh + r_h * (a - h * (r_h.square() * (a * h).mean(-1, keepdim=True)))
    du = s["scale"] * gate * dh
    b = du * post
    df = r_f * (b - f * (r_f.square() * (b * f).mean(-1, keepdim=True)))
    dgate = (s["scale"] * u * dh).view(n, case["gates"], rows, D).sum(2)
    out.update(dx=dh.to(dtype), df=df.to(dtype), dgate=dgate.to(dtype), dpost=(du * f * r_f).sum(1).to(dtype), dpre=(dy * h * r_h).sum(1).to(dtype))
    return out


def _plain(s):
    op = s["case"]["op"]
    if op == "loss":
        return _loss_plain(s)
    if op == "norm":
        return _norm_plain(s)
    if op == "pack":
        return {"x": _dequantise(*_quantise(s["x"])).to(s["x"].dtype)}
    x = _dequantise(s["codes"][:, :, : s["case"]["D"]], s["scales"])
    return {"dweight": torch.bmm(s["dy"].float().transpose(1, 2), x).to(s["dy"].dtype)}


# ------------------------------------------------------------------------------------------------------ the package's calls
def _package(s):
    from paper_1810_07766_b200 import ops

    case, op = s["case"], s["case"]["op"]
    if op == "loss":
        if not case["train"]:
            loss, lse = ops.linear_cross_entropy_forward(s["hidden"], s["weight"], s["targets"], ignore_index=IGNORE, reduction="none")
            return {"loss": loss, "lse": lse}
        loss, lse = ops.linear_cross_entropy_forward(s["hidden"], s["weight"], s["targets"], ignore_index=IGNORE, reduction="mean")
        dhidden, dweight = ops.linear_cross_entropy_backward(s["dloss"], s["hidden"], s["weight"], s["targets"], lse, ignore_index=IGNORE, reduction="mean")
        return {"loss": loss, "dhidden": dhidden, "dweight": dweight}
    if op == "norm":
        h, y, kept = ops.gated_residual_norm_forward(s["x"], s["f"], s["gate"], s["post"], s["pre"], scale=s["scale"], eps=EPS, keep=case["keep"])
        if not case["train"]:
            return {"h": h, "y": y}
        dx, df, dgate, dpost, dpre = ops.gated_residual_norm_backward(s["dh"], s["dy"], kept, s["gate"], s["post"], s["pre"], scale=s["scale"])
        return {"h": h, "y": y, "dx": dx, "df": df, "dgate": dgate, "dpost": dpost, "dpre": dpre}
    if op == "pack":
        return {"x": ops.unpack_activation(ops.pack_activation(s["x"]))}
    kept = ops.PackedActivation(s["codes"], s["scales"], case["D"], s["dy"].dtype)
    return {"dweight": ops.packed_weight_grad(s["dy"], kept)}


def run(state):
    return _package(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------------------------- work
def work(case):
    """Each input read once, each output written once; the products that the definition has (the logits made once)."""
    e = 4 if case["dtype"] == "f32" else 2
    n, T, D = case["n"], case["T"], case["D"]
    if case["op"] == "loss":
        V, valid = case["V"], T - int(case["ignored"] * T)
        if not case["train"]:
            return {"bytes": n * (e * (valid * D + V * D) + 16 * T), "flops": 2 * n * valid * V * D}
        return {"bytes": n * (e * (valid * D + 2 * V * D + T * D) + 8 * T + 8), "flops": 6 * n * valid * V * D}
    if case["op"] == "norm":
        rest = n * D * e * (case["gates"] + 2)
        if not case["train"]:
            return {"bytes": 4 * n * T * D * e + rest, "flops": 12 * n * T * D}
        # forward: x, f in, h, y out; backward: dh, dy in, dx, df out, and what was kept: h and f again, or an 8-bit copy of each, written and read
        kept = 4 * n * T * D if case["keep"] == "int8" else 2 * n * T * D * e
        return {"bytes": 8 * n * T * D * e + kept + 3 * rest, "flops": 40 * n * T * D}
    codes = n * T * (D + 4 * -(-D // GROUP))
    if case["op"] == "pack":
        return {"bytes": 2 * n * T * D * e + 2 * codes, "flops": 4 * n * T * D}
    return {"bytes": codes + n * e * (T * case["V"] + case["V"] * D), "flops": 2 * n * T * case["V"] * D}


# ------------------------------------------------------------------------------------------------- definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op, n, T, D = case["op"], case["n"], case["T"], case["D"]
    if op == "loss":
        h, w, y = s["hidden"].double(), s["weight"].double(), s["targets"]
        each, total = (torch.zeros(n, T, dtype=torch.float64, device="cuda") for _ in range(2))
        dh, dw = torch.zeros_like(h), torch.zeros_like(w)
        mean = torch.zeros(n, dtype=torch.float64, device="cuda")
        for i in range(n):
            keep = torch.nonzero(y[i] != IGNORE).flatten()
            if not len(keep):
                continue
            k = torch.arange(len(keep), device="cuda")
            z = h[i, keep] @ w[i].T
            lse = torch.logsumexp(z, dim=1)
            total[i, keep] = lse
            each[i, keep] = lse - z[k, y[i, keep]]
            mean[i] = each[i].sum() / len(keep)
            if case["train"]:
                z = torch.exp(z - lse[:, None])
                z[k, y[i, keep]] -= 1.0
                z *= s["dloss"][i].double() / len(keep)
                dh[i, keep] = z @ w[i]
                dw[i] = z.T @ h[i, keep]
        return {"loss": mean, "dhidden": dh, "dweight": dw} if case["train"] else {"loss": each, "lse": total}
    if op == "norm":
        x, f, post, pre = (s[k].double() for k in ("x", "f", "post", "pre"))
        post, pre = post.unsqueeze(1), pre.unsqueeze(1)
        index = torch.arange(T, device="cuda") // (T // case["gates"])
        gate = s["gate"].double()[:, index] * s["scale"]

        def unit(z):
            return 1.0 / torch.sqrt((z * z).sum(-1, keepdim=True) / D + EPS)

        rf = unit(f)
        h = x + gate * f * rf * post
        rh = unit(h)
        out = {"h": h, "y": pre * rh * h}
        if not case["train"]:
            return out
        if case["keep"] == "int8":
            f, h = _kept(f), _kept(h.to(s["x"].dtype).double())

        def through(d, z, r):  # gradient of z * r(z) against d
            zn = z * r
            return r * (d - zn * (d * zn).sum(-1, keepdim=True) / D)

        dy = s["dy"].double()
        t = s["dh"].double() + through(dy * pre, h, rh)
        dgate = torch.zeros(n, case["gates"], D, dtype=torch.float64, device="cuda")
        dgate.index_add_(1, index, s["scale"] * t * f * rf * post)
        out.update(dx=t, df=through(t * gate * post, f, rf), dgate=dgate, dpost=torch.einsum("ntd,ntd->nd", t * gate, f * rf), dpre=torch.einsum("ntd,ntd->nd", dy, h * rh))
        return out
    if op == "pack":
        return {"x": _kept(s["x"].double())}
    width = torch.arange(D, device="cuda") // GROUP
    x = s["codes"][:, :, :D].double() * s["scales"].double()[:, :, width]
    return {"dweight": torch.einsum("nto,nti->noi", s["dy"].double(), x)}


def _kept(x):
    """Values that stand for x after 8 bits: the scale of a group of columns, and the factor that gives the codes, are held in float32."""
    parts = []
    for part in x.split(GROUP, dim=-1):
        top = part.abs().amax(-1, keepdim=True)
        factor = torch.where(top > 0, 127.0 / top, 0.0).float().double()
        parts.append(torch.round((part * factor).float().double()) * (top / 127.0).float().double())
    return torch.cat(parts, dim=-1)
