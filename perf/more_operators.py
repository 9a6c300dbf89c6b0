"""What a further set of training operators is measured on: cases, inputs, a plain form of each operator in elementary torch
operations, the calls of the package that compute the same, and a definition in 64 bits to hold both against.

The package simulates ``n`` workers on one GPU, so every operator has a leading worker axis.  Three operators, the parts of a worker's
language model before, between and after its blocks:

* ``embed``: rows of a table looked up by token and scaled, and the table's gradient (written whole, or added to what is there);
* ``mix``: linear attention with a decay for each head over sequences (forward, or forward and backward), and ``step``: its
  recurrent form for one new token of each sequence;
* ``distil``: the divergence of the softmax of ``hidden @ weight.T`` from a teacher's kept logits, with its gradient.
"""
import math

import torch

own = False

IGNORE = -100
CHUNK = 64
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # four workers' short batches over a small vocabulary: every call is launch latency
        {"name": "embed 4x32 of 1000x256 bf16", "op": "embed", "dtype": "bf16", "n": 4, "T": 32, "V": 1000, "D": 256, "train": True, "add": False, "ignored": 0.0},
        # eight workers in full precision, a table shared with the output layer, whose gradient is already there; a quarter is padding
        {"name": "embed 8x4000 of 10001x650 f32 tied", "op": "embed", "dtype": "f32", "n": 8, "T": 4000, "V": 10001, "D": 650, "train": True, "add": True, "ignored": 0.25},
        # a long batch over a large vocabulary
        {"name": "embed 32768 of 131072x2048 bf16", "op": "embed", "dtype": "bf16", "n": 1, "T": 32768, "V": 131072, "D": 2048, "train": True, "add": False, "ignored": 0.0},
        # one new token of each of eight sequences: latency
        {"name": "step 8x4x64x64 bf16", "op": "step", "dtype": "bf16", "n": 1, "B": 8, "H": 4, "K": 64, "W": 64},
        # text generated for many sequences at once
        {"name": "step 128x16x128x128 bf16", "op": "step", "dtype": "bf16", "n": 1, "B": 128, "H": 16, "K": 128, "W": 128},
        # four workers' training step in full precision, sizes that no tile divides
        {"name": "mix 4x3x333x5x48x40 f32", "op": "mix", "dtype": "f32", "n": 4, "B": 3, "T": 333, "H": 5, "K": 48, "W": 40, "train": True, "ragged": False},
        # a prompt read in one pass: few heads, many tokens
        {"name": "mix prompt 65536x8x64x64 bf16", "op": "mix", "dtype": "bf16", "n": 1, "B": 1, "T": 65536, "H": 8, "K": 64, "W": 64, "train": False, "ragged": False},
        # two workers' training step over padded sequences
        {"name": "mix 2x8x2048x16x128x128 bf16", "op": "mix", "dtype": "bf16", "n": 2, "B": 8, "T": 2048, "H": 16, "K": 128, "W": 128, "train": True, "ragged": True},
        # four workers with a small vocabulary and one short batch each
        {"name": "distil 4x32x1000 top 8 bf16", "op": "distil", "dtype": "bf16", "n": 4, "T": 32, "V": 1000, "D": 256, "k": 8, "tau": 1.0, "train": True, "ignored": 0.0},
        # eight workers on full-precision replicas, sizes that no tile divides; a quarter of the tokens is padding
        {"name": "distil 8x500x10001 top 20 f32", "op": "distil", "dtype": "f32", "n": 8, "T": 500, "V": 10001, "D": 650, "k": 20, "tau": 2.0, "train": True, "ignored": 0.25},
        # how far a student is from its teacher, token by token
        {"name": "distil eval 2048x50001 top 50 bf16", "op": "distil", "dtype": "bf16", "n": 1, "T": 2048, "V": 50001, "D": 1024, "k": 50, "tau": 1.0, "train": False, "ignored": 0.0},
        # the largest: a long batch over a large vocabulary, prompts left out
        {"name": "distil 4096x131072 top 64 bf16", "op": "distil", "dtype": "bf16", "n": 1, "T": 4096, "V": 131072, "D": 2048, "k": 64, "tau": 2.0, "train": True, "ignored": 0.1},
    ]


def _log_uniform(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    largest = max(work(c)["flops"] for c in listed())
    op = rng.choice(["embed", "embed", "mix", "mix", "mix", "step", "distil", "distil"])
    while True:
        dtype = rng.choice(["bf16", "f32"])
        n = rng.choice([1, 1, 2, 3, 4, 8])
        if op == "embed":
            c = {"op": op, "dtype": dtype, "n": n, "T": _log_uniform(rng, 1, 65536), "V": _log_uniform(rng, 100, 131072), "D": _log_uniform(rng, 64, 8192),
                 "train": rng.random() < 0.8, "add": rng.random() < 0.4, "ignored": rng.choice([0.0, 0.1, 0.5])}
            if n * c["T"] * c["D"] <= 70_000_000 and n * c["V"] * c["D"] <= 270_000_000:
                return c
        elif op == "step":
            c = {"op": op, "dtype": dtype, "n": n, "B": _log_uniform(rng, 1, 256), "H": _log_uniform(rng, 1, 32), "K": rng.randint(8, 128), "W": rng.randint(8, 128)}
            if n * c["B"] * c["H"] * c["K"] * c["W"] <= 34_000_000:
                return c
        elif op == "mix":
            even = rng.random() < 0.5
            c = {"op": op, "dtype": dtype, "n": n, "B": _log_uniform(rng, 1, 16), "T": _log_uniform(rng, 1, 65536), "H": _log_uniform(rng, 1, 32),
                 "K": rng.choice([32, 64, 128]) if even else rng.randint(8, 128), "W": rng.choice([32, 64, 128]) if even else rng.randint(8, 128),
                 "train": rng.random() < 0.7, "ragged": rng.random() < 0.4}
            if n * c["B"] * c["T"] * c["H"] * max(c["K"], c["W"]) <= 67_000_000:
                return c
        else:
            V = _log_uniform(rng, 100, 131072)
            c = {"op": op, "dtype": dtype, "n": n, "T": _log_uniform(rng, 1, 8192), "V": V, "D": _log_uniform(rng, 64, 4096), "k": _log_uniform(rng, 1, 100),
                 "tau": rng.choice([1.0, 2.0, 3.5]), "train": rng.random() < 0.7, "ignored": rng.choice([0.0, 0.1, 0.5])}
            if n * c["T"] * c["D"] > 200_000_000 or n * c["T"] * V > 4096 * 131072 or n * V * c["D"] > 300_000_000:
                continue
            if work(c)["flops"] <= (largest if dtype == "bf16" else largest / 8):
                return c


# --------------------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype = _TYPES[case["dtype"]]
    n = case["n"]

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    s = {"case": case}
    if case["op"] == "embed":
        T, V, D = case["T"], case["V"], case["D"]
        s["weight"] = normal(n, V, D, scale=1.0 / math.sqrt(D))
        s["scale"] = math.sqrt(D)
        # frequent words have small numbers
        tokens = (torch.exp(uniform(n, T).double() * math.log(V + 1)) - 1).long().clamp(0, V - 1)
        s["tokens"] = torch.where(uniform(n, T) < case["ignored"], IGNORE, tokens)
        if case["train"]:
            s["dout"] = normal(n, T, D)
            if case["add"]:
                s["there"] = normal(n, V, D)
                s["dweight"] = torch.empty_like(s["there"])
        return s
    if case["op"] in ("mix", "step"):
        B, H, K, W = case["B"], case["H"], case["K"], case["W"]
        tokens = (case["T"],) if case["op"] == "mix" else ()
        # queries, keys and values are parts of one projection's output
        joint = normal(n, B, *tokens, H, 2 * K + W)
        s["q"], s["k"], s["v"] = joint[..., :K], joint[..., K:2 * K], joint[..., 2 * K:]
        # from heads that forget within a few tokens to heads that remember a thousand
        spread = 2.0 + 8.0 * (torch.arange(H, device="cuda") + uniform(n, H)) / H
        s["log_decay"] = torch.log1p(-torch.exp2(-spread))
        s["scale"] = 1.0 / math.sqrt(K)
        s["state"] = torch.randn(n, B, H, K, W, generator=g, device="cuda")
        if case["op"] == "step":
            s["next"] = torch.empty_like(s["state"])
            return s
        s["lengths"] = (uniform(n, B) * (case["T"] + 1)).long().clamp(0, case["T"]) if case["ragged"] else None
        if case["train"]:
            s["dout"] = normal(n, B, case["T"], H, W)
            s["dstate"] = torch.randn(n, B, H, K, W, generator=g, device="cuda")
        return s
    T, V, D, k = case["T"], case["V"], case["D"], case["k"]
    s["hidden"] = normal(n, T, D)
    s["weight"] = normal(n, V, D, scale=2.0 / math.sqrt(D))
    # different words for each token, their logits in falling order; of some tokens the teacher kept fewer
    first = (uniform(n, T, 1).double() * V).long()
    apart = 1 + (uniform(n, T, 1).double() * (V // k)).long().clamp(0, V // k - 1)
    ids = (first + torch.arange(k, device="cuda") * apart) % V
    logits = 12.0 - torch.cumsum(-torch.log(uniform(n, T, k).clamp(min=1e-6)) * (8.0 / k), -1)
    kept = torch.where(uniform(n, T, 1) < 0.2, (uniform(n, T, 1) * k).long() + 1, k)
    kept = torch.where(uniform(n, T, 1) < case["ignored"], 0, kept)
    s["top_ids"] = torch.where(torch.arange(k, device="cuda") < kept, ids, IGNORE)
    s["top_logits"] = logits.to(dtype)
    s["dloss"] = uniform(n) + 0.5 if case["train"] else None
    return s


# ---------------------------------------------------------------------------------------------------------- plain forms
def _embed_plain(s):
    case, dtype, tokens = s["case"], s["weight"].dtype, s["tokens"]
    n, V, D = s["weight"].shape
    valid = tokens != IGNORE
    worker = torch.arange(n, device="cuda")[:, None]
    rows = s["weight"][worker, tokens.clamp(min=0)].float() * s["scale"]
    out = {"out": torch.where(valid[..., None], rows, 0.0).to(dtype)}
    if case["train"]:
        total = torch.zeros(n * V, D, device="cuda")
        place = (worker * V + tokens)[valid]
        total.index_add_(0, place, s["dout"].float()[valid])
        total = total.view(n, V, D) * s["scale"]
        out["dweight"] = (s["there"].float() + total if case["add"] else total).to(dtype)
    return out


def _heads_first(x):
    """[n, B, T, H, d] as 32-bit [n * B, H, T, d]."""
    return x.float().flatten(0, 1).transpose(1, 2)


def _tokens_first(x, n):
    return x.transpose(1, 2).unflatten(0, (n, -1))


def _mix_plain(s):
    case, dtype = s["case"], s["q"].dtype
    n, B, T, H, K = s["q"].shape
    scale = s["scale"]
    q, k, v = (_heads_first(s[x]) for x in "qkv")
    rate = s["log_decay"].double().repeat_interleave(B, 0)
    length = torch.full((n * B,), T, device="cuda") if s["lengths"] is None else s["lengths"].flatten()
    there = (torch.arange(T, device="cuda") < length[:, None])[:, None, :, None]
    q, k, v = (torch.where(there, x, 0.0) for x in (q, k, v))
    state = s["state"].flatten(0, 1)
    out = torch.zeros_like(v)

    def decays(t0, size):
        """Of a chunk: from token to token, from the state before it to each token, from each token to its end, over all of it."""
        i = torch.arange(size, device="cuda")
        inside = (length - t0).clamp(0, size)
        apart = i[:, None] - i
        between = torch.where(apart >= 0, torch.exp(rate[..., None, None] * apart.clamp(min=0)), 0.0)
        since = torch.exp(rate[..., None] * (i + 1))[..., None]
        left = (inside[:, None] - 1 - i)[:, None]
        until = torch.where(left >= 0, torch.exp(rate[..., None] * left.clamp(min=0)), 0.0)[..., None]
        whole = torch.exp(rate * inside[:, None])[..., None, None]
        return between.float(), since.float(), until.float(), whole.float()

    before = []
    for t0 in range(0, T, CHUNK):
        part = slice(t0, min(t0 + CHUNK, T))
        qc, kc, vc = q[:, :, part], k[:, :, part], v[:, :, part]
        between, since, until, whole = decays(t0, qc.shape[2])
        before.append(state)
        scores = (qc @ kc.mT) * between
        out[:, :, part] = scale * (scores @ vc + since * (qc @ state))
        state = whole * state + (kc * until).mT @ vc
    result = {"out": _tokens_first(out, n).to(dtype), "state": state.unflatten(0, (n, B))}
    if not case["train"]:
        return result
    do = torch.where(there, _heads_first(s["dout"]), 0.0)
    later = s["dstate"].flatten(0, 1)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for t0 in reversed(range(0, T, CHUNK)):
        part = slice(t0, min(t0 + CHUNK, T))
        qc, kc, vc, dc = q[:, :, part], k[:, :, part], v[:, :, part], do[:, :, part]
        between, since, until, whole = decays(t0, qc.shape[2])
        state = before[t0 // CHUNK]
        scores = scale * (qc @ kc.mT) * between
        dscores = scale * (dc @ vc.mT) * between
        dq[:, :, part] = dscores @ kc + scale * since * (dc @ state.mT)
        dk[:, :, part] = dscores.mT @ qc + until * (vc @ later.mT)
        dv[:, :, part] = scores.mT @ dc + until * (kc @ later)
        later = whole * later + scale * (qc * since).mT @ dc
    result.update({name: _tokens_first(x, n).to(dtype) for name, x in (("dq", dq), ("dk", dk), ("dv", dv))})
    result["dstate"] = later.unflatten(0, (n, B))
    return result


def _step_plain(s):
    decay = torch.exp(s["log_decay"].double()).float()[:, None, :, None, None]
    q, k, v = (s[x].float() for x in "qkv")
    state = decay * s["state"] + k[..., :, None] * v[..., None, :]
    return {"out": (s["scale"] * (q[..., :, None] * state).sum(-2)).to(s["q"].dtype), "state": state}


def _teacher(s):
    """Probabilities of the teacher's kept words and their logarithms, zero where nothing is kept; which tokens take part."""
    kept = s["top_ids"] != IGNORE
    x = torch.where(kept, s["top_logits"].float() / s["case"]["tau"], -math.inf)
    valid = kept.any(-1)
    top = torch.where(valid[..., None], x.amax(-1, keepdim=True), 0.0)
    e = torch.exp(x - top)
    total = torch.where(valid[..., None], e.sum(-1, keepdim=True), 1.0)
    return e / total, torch.where(kept, x - top - total.log(), 0.0), valid


def _distil_plain(s):
    case, dtype, tau = s["case"], s["hidden"].dtype, s["case"]["tau"]
    h, w = s["hidden"].float(), s["weight"].float()
    prob, log_prob, valid = _teacher(s)
    at = s["top_ids"].clamp(min=0)
    z = torch.bmm(h, w.transpose(1, 2)).div_(tau)
    top = z.amax(-1, keepdim=True)
    hit = z.gather(-1, at)
    e = z.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    lse = top + total.log()
    each = tau * tau * (prob * (log_prob - (hit - lse))).sum(-1)
    if not case["train"]:
        return {"loss": each, "lse": torch.where(valid, tau * lse.squeeze(-1), 0.0)}
    count = valid.sum(-1).clamp(min=1).float()
    c = torch.where(valid, (tau * s["dloss"] / count)[:, None], 0.0)[..., None]
    dl = e.mul_(c / total)
    dl.scatter_add_(-1, at, -c * prob)
    return {"loss": each.sum(-1) / count, "dhidden": torch.bmm(dl, w).to(dtype), "dweight": torch.bmm(dl.transpose(1, 2), h).to(dtype)}


_PLAIN = {"embed": _embed_plain, "mix": _mix_plain, "step": _step_plain, "distil": _distil_plain}


# ------------------------------------------------------------------------------------------------------ the package's calls
def _package(s):
    from paper_1810_07766_b200 import ops

    case, op = s["case"], s["case"]["op"]
    if op == "embed":
        out = {"out": ops.embedding_forward(s["tokens"], s["weight"], scale=s["scale"], ignore_index=IGNORE)}
        if case["train"]:
            if case["add"]:
                # the gradient that the output layer has left there
                s["dweight"].copy_(s["there"])
                out["dweight"] = ops.embedding_backward(s["dout"], s["tokens"], case["V"], scale=s["scale"], ignore_index=IGNORE, dweight=s["dweight"], accumulate=True)
            else:
                out["dweight"] = ops.embedding_backward(s["dout"], s["tokens"], case["V"], scale=s["scale"], ignore_index=IGNORE)
        return out
    if op == "step":
        out = ops.linear_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"], scale=s["scale"], new_state=s["next"])
        return {"out": out, "state": s["next"]}
    if op == "mix":
        out, state = ops.linear_attention_forward(s["q"], s["k"], s["v"], s["log_decay"], scale=s["scale"], state=s["state"], lengths=s["lengths"])
        if not case["train"]:
            return {"out": out, "state": state}
        dq, dk, dv, dstate = ops.linear_attention_backward(s["dout"], s["dstate"], s["q"], s["k"], s["v"], s["log_decay"], scale=s["scale"], state=s["state"],
                                                           lengths=s["lengths"])
        return {"out": out, "state": state, "dq": dq, "dk": dk, "dv": dv, "dstate": dstate}
    teacher = {"temperature": case["tau"], "ignore_index": IGNORE, "reduction": "mean" if case["train"] else "none"}
    loss, lse = ops.linear_distillation_forward(s["hidden"], s["weight"], s["top_ids"], s["top_logits"], **teacher)
    if not case["train"]:
        return {"loss": loss, "lse": lse}
    dhidden, dweight = ops.linear_distillation_backward(s["dloss"], s["hidden"], s["weight"], s["top_ids"], s["top_logits"], lse, **teacher)
    return {"loss": loss, "dhidden": dhidden, "dweight": dweight}


def run(state):
    return _package(state) if own else _PLAIN[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------------------------- work
def work(case):
    """Each input read once, each output written once; the operations that the definition has (attention in its recurrent form, the
    logits made once)."""
    e = 4 if case["dtype"] == "f32" else 2
    n, op = case["n"], case["op"]
    if op == "embed":
        T, V, D = case["T"], case["V"], case["D"]
        valid = T * (1.0 - case["ignored"])
        forward = {"bytes": int(n * (min(valid, V) * D * e + T * (D * e + 8))), "flops": int(n * valid * D)}
        if not case["train"]:
            return forward
        table = (2 if case["add"] else 1) * n * V * D * e
        return {"bytes": int(forward["bytes"] + n * T * 8 + n * valid * D * e + table), "flops": int(forward["flops"] + n * (valid + V) * D)}
    if op in ("mix", "step"):
        B, H, K, W = case["B"], case["H"], case["K"], case["W"]
        states, tokens = n * B * H * K * W * 4, n * B * H * case.get("T", 1)
        if case.get("ragged"):
            tokens //= 2  # lengths are spread evenly
        if op == "step" or not case["train"]:
            return {"bytes": tokens * (2 * K + 2 * W) * e + 2 * states, "flops": 5 * tokens * K * W}
        return {"bytes": tokens * (2 * K + 2 * W) * e + 2 * states + tokens * (4 * K + 3 * W) * e + 3 * states, "flops": 19 * tokens * K * W}
    T, V, D, k = case["T"], case["V"], case["D"], case["k"]
    valid = T * (1.0 - case["ignored"])
    teacher = n * T * k * (8 + e)
    if not case["train"]:
        return {"bytes": int(n * (e * (valid * D + V * D) + 8 * T) + teacher), "flops": int(2 * n * valid * V * D)}
    return {"bytes": int(n * (e * (valid * D + 2 * V * D + T * D) + 8) + teacher), "flops": int(6 * n * valid * V * D)}


# ------------------------------------------------------------------------------------------------- definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _embed_exact, "mix": _mix_exact, "step": _step_exact, "distil": _distil_exact}[case["op"]](case, s)


def _embed_exact(case, s):
    n, T, V, D = case["n"], case["T"], case["V"], case["D"]
    out = {"out": torch.zeros(n, T, D, dtype=torch.float64, device="cuda")}
    grads = torch.zeros(n, V, D, dtype=torch.float64, device="cuda") if case["train"] else None
    for w in range(n):
        at = torch.nonzero(s["tokens"][w] != IGNORE).flatten()
        words = s["tokens"][w, at]
        out["out"][w, at] = s["weight"][w].double()[words] * s["scale"]
        if case["train"]:
            words, order = torch.sort(words)
            sums = torch.cumsum(s["dout"][w, at[order]].double(), 0)
            last = torch.nonzero(torch.cat([words[1:] != words[:-1], words.new_ones(min(1, len(words)), dtype=torch.bool)])).flatten()
            upto = sums[last]
            grads[w, words[last]] = torch.diff(upto, dim=0, prepend=torch.zeros_like(upto[:1])) * s["scale"]
    if case["train"]:
        out["dweight"] = grads + s["there"].double() if case["add"] else grads
    return out


def _mix_exact(case, s):
    """Token by token."""
    n, B, T, H, K, W = (case[x] for x in ("n", "B", "T", "H", "K", "W"))
    elements = n * B * H * K * W
    if T * (2 if case["train"] else 1) * (60e-6 + elements * 8 * 12 / 4e12) > 15:
        return None
    q, k, v = (s[x].double() for x in "qkv")
    length = torch.full((n, B), T, device="cuda") if s["lengths"] is None else s["lengths"]
    decay = torch.exp(s["log_decay"].double())[:, None, :, None, None]
    active = (torch.arange(T, device="cuda")[:, None, None] < length).double()[..., None, None, None]  # [T, n, B, 1, 1, 1]
    on = active[..., 0].permute(1, 2, 0, 3, 4)
    q, k, v = q * on, k * on, v * on
    rates = torch.where(active > 0, decay, 1.0)
    S = s["state"].double()
    out, scale = torch.zeros_like(v), s["scale"]
    do, dq = (s["dout"].double() * on, torch.zeros_like(q)) if case["train"] else (None, None)
    for t in range(T):
        S = S * rates[t]
        S.addcmul_(k[:, :, t, :, :, None], v[:, :, t, :, None, :])
        out[:, :, t] = (q[:, :, t, :, :, None] * S).sum(-2) * scale
        if case["train"]:
            dq[:, :, t] = (do[:, :, t, :, None, :] * S).sum(-1) * scale
    result = {"out": out, "state": S}
    if case["train"]:
        R = s["dstate"].double()
        dk, dv = torch.zeros_like(k), torch.zeros_like(v)
        for t in range(T - 1, -1, -1):
            R = torch.addcmul(R, q[:, :, t, :, :, None], do[:, :, t, :, None, :], value=scale)
            dk[:, :, t] = (R * v[:, :, t, :, None, :]).sum(-1)
            dv[:, :, t] = (R * k[:, :, t, :, :, None]).sum(-2)
            R *= rates[t]
        result.update(dq=dq, dk=dk * on, dv=dv * on, dstate=R)
    return result


def _step_exact(case, s):
    q, k, v = (s[x].double() for x in "qkv")
    S = s["state"].double() * torch.exp(s["log_decay"].double())[:, None, :, None, None] + torch.einsum("nbhk,nbhw->nbhkw", k, v)
    return {"out": torch.einsum("nbhk,nbhkw->nbhw", q, S) * s["scale"], "state": S}


def _distil_exact(case, s):
    n, T, tau = case["n"], case["T"], case["tau"]
    h, w = s["hidden"].double(), s["weight"].double()
    each, lses = (torch.zeros(n, T, dtype=torch.float64, device="cuda") for _ in range(2))
    mean = torch.zeros(n, dtype=torch.float64, device="cuda")
    dh, dw = torch.zeros_like(h), torch.zeros_like(w)
    for i in range(n):
        keep = torch.nonzero((s["top_ids"][i] != IGNORE).any(-1)).flatten()
        if not len(keep):
            continue
        ids = s["top_ids"][i, keep]
        logits = s["top_logits"][i, keep].double().masked_fill(ids == IGNORE, -math.inf) / tau
        log_q = torch.log_softmax(logits, -1).masked_fill(ids == IGNORE, 0.0)
        q = torch.softmax(logits, -1)
        ids = ids.clamp(min=0)
        z = h[i, keep] @ w[i].T / tau
        lse = torch.logsumexp(z, 1, keepdim=True)
        lses[i, keep] = tau * lse[:, 0]
        each[i, keep] = tau * tau * (q * (log_q - z.gather(1, ids) + lse)).sum(1)
        mean[i] = each[i].sum() / len(keep)
        if case["train"]:
            dz = torch.exp(z - lse).scatter_add_(1, ids, -q) * (tau * s["dloss"][i].double() / len(keep))
            dh[i, keep], dw[i] = dz @ w[i], dz.T @ h[i, keep]
    return {"loss": mean, "dhidden": dh, "dweight": dw} if case["train"] else {"loss": each, "lse": lses}
