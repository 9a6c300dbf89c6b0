"""Training operators next to the RPS step: the gradient of a worker's own step, for all workers in one call.

A thin layer over the C ABI of ``include/rps_ops.h``: argument checks, outputs and workspaces (PyTorch lends the device
memory and the current stream), nothing else.  Every operator takes its tensors with a leading worker axis (``[n, ...]``) or
without one (a single worker), in float32 or bfloat16, one type for all tensors of a call.  Parameters may be views
into the rows of an ``[n][pitch]`` array such as ``RPS.x_dev``: only the innermost axis has to be contiguous.

* ``linear_cross_entropy``: softmax cross entropy of ``hidden @ weight.T`` over a large vocabulary without keeping the logits;
* ``gated_residual_norm``: norm after a block, gate, residual scale, residual sum, norm before the next block;
* ``pack_activation`` / ``unpack_activation`` / ``packed_weight_grad``: activations kept in 8 bits, and their use in the
  backward pass (``gated_residual_norm(..., keep="int8")``, ``linear_8bit``).

The functions named ``*_forward`` and ``*_backward`` are single calls of the library; the names without a suffix are
differentiable.  There is no CPU fallback: a missing library, a CPU tensor or a failing call raises.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional, Tuple

import torch

from . import binding
from .binding import RPS_BF16, RPS_F32, RPS_OK, RPSError

GROUP = 128               # columns that share a scale in 8-bit activations (RPS_PACK_GROUP)
MAX_NORM_COLS = 16384     # RPS_MAX_NORM_COLS
_REDUCTION = {"none": 0, "sum": 1, "mean": 2}
_DTYPE = {torch.float32: RPS_F32, torch.bfloat16: RPS_BF16}

# every symbol include/rps_ops.h declares
SYMBOLS = (
    "rps_lce_workspace", "rps_lce_forward", "rps_lce_backward", "rps_norm_forward", "rps_norm_workspace",
    "rps_norm_backward", "rps_pack_pitch", "rps_pack", "rps_unpack", "rps_wgrad_workspace", "rps_packed_wgrad",
    "rps_ops_check", "rps_ops_last_error",
)

_i32, _i64, _dbl = ctypes.c_int32, ctypes.c_int64, ctypes.c_double


class rps_lce_desc(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("reduction", _i32), ("n", _i32), ("tokens", _i64), ("vocab", _i64), ("cols", _i64),
                ("ignore_index", _i64), ("hidden_row", _i64), ("hidden_worker", _i64), ("weight_row", _i64),
                ("weight_worker", _i64), ("dweight_row", _i64), ("dweight_worker", _i64)]


class rps_norm_desc(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("n", _i32), ("tokens", _i64), ("cols", _i64), ("gates", _i64), ("post_worker", _i64),
                ("pre_worker", _i64), ("gate_worker", _i64), ("scale", _dbl), ("eps", _dbl), ("wait_limit_ms", _i32),
                ("withhold_sums", _i32)]


class rps_wgrad_desc(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("n", _i32), ("tokens", _i64), ("outs", _i64), ("cols", _i64), ("dy_row", _i64),
                ("dy_worker", _i64), ("dweight_row", _i64), ("dweight_worker", _i64), ("wait_limit_ms", _i32),
                ("withhold_copies", _i32)]


_lib = None


def _library() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        lib = binding.load_library()
        vp, cint, size = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        lce, norm, wgrad = (ctypes.POINTER(t) for t in (rps_lce_desc, rps_norm_desc, rps_wgrad_desc))
        sizep = ctypes.POINTER(size)
        sig = {
            "rps_lce_workspace": (cint, [lce, vp, cint, sizep]),
            "rps_lce_forward": (cint, [lce] + [vp] * 6 + [size, vp]),
            "rps_lce_backward": (cint, [lce] + [vp] * 8 + [size, vp]),
            "rps_norm_forward": (cint, [norm] + [vp] * 14),
            "rps_norm_workspace": (cint, [norm, sizep]),
            "rps_norm_backward": (cint, [norm] + [vp] * 17 + [size, vp]),
            "rps_pack_pitch": (_i64, [_i64]),
            "rps_pack": (cint, [cint, _i64, _i64, vp, _i64, vp, vp, vp]),
            "rps_unpack": (cint, [cint, _i64, _i64, vp, vp, vp, _i64, vp]),
            "rps_wgrad_workspace": (cint, [wgrad, vp, sizep]),
            "rps_packed_wgrad": (cint, [wgrad] + [vp] * 5 + [size, vp]),
            "rps_ops_check": (cint, [vp]),
            "rps_ops_last_error": (ctypes.c_char_p, []),
        }
        for name, (res, args) in sig.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def _call(name: str, device: int, *args) -> None:
    """One call of the library with the tensors' device current."""
    lib = _lib or _library()
    if torch.cuda.current_device() == device:
        rc = getattr(lib, name)(*args)
    else:
        with torch.cuda.device(device):
            rc = getattr(lib, name)(*args)
    if rc != RPS_OK:
        raise RPSError(rc, name, lib.rps_ops_last_error().decode())


# What a call says about its arguments' types, shapes and strides is checked and described to the library once; the checked
# descriptions are kept by exactly those (never by an address or a value), as a small call's time is mostly such work.
_plans: dict = {}
_MOST_PLANS = 4096


def _keep(key, plan):
    if len(_plans) >= _MOST_PLANS:
        _plans.clear()
    _plans[key] = plan
    return plan


def _device_of(**tensors) -> int:
    """Index of the one CUDA device that all of them are on."""
    device = -1
    for name, t in tensors.items():
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise ValueError(f"{name} must be a CUDA tensor")
        if device < 0:
            device = t.get_device()
        elif t.get_device() != device:
            raise ValueError(f"{name} must be on the device of the other tensors")
    return device


def check(device: Optional[torch.device] = None) -> None:
    """Synchronises the current stream of the device and raises if a kernel of an earlier call gave up (``rps_ops_check``)."""
    index = torch.cuda.current_device() if device is None else torch.empty(0, device=device).get_device()
    _call("rps_ops_check", index, _stream(index))


def _stream(device: int) -> int:
    return torch._C._cuda_getCurrentRawStream(device)


def _dense_layout(shape) -> Tuple[Tuple[int, ...], Tuple[int, ...]]:
    """(shape, strides) of a contiguous tensor: torch.empty_strided takes them in two thirds of torch.empty's time."""
    strides, step = [], 1
    for size in reversed(tuple(shape)):
        strides.append(step)
        step *= max(size, 1)
    return tuple(shape), tuple(reversed(strides))


def _new(layout, dtype: torch.dtype, device: torch.device) -> torch.Tensor:
    # torch's allocations start on 512-byte boundaries; memory of the current stream goes back to it when the tensor is dropped
    return torch.empty_strided(layout[0], layout[1], dtype=dtype, device=device)


def _check(name: str, t: torch.Tensor, like: Optional[torch.Tensor], shape: Tuple[int, ...]) -> None:
    if t.dtype not in _DTYPE:
        raise ValueError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    if like is not None and t.dtype != like.dtype:
        raise ValueError(f"{name} must have the type of the other tensors ({like.dtype})")
    if tuple(t.shape) != shape:
        raise ValueError(f"{name} must have shape {shape}, not {tuple(t.shape)}")


def _dense(name: str, t: torch.Tensor) -> None:
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _matrix_strides(name: str, t: torch.Tensor) -> Tuple[int, int]:
    """(row, worker) strides of a [..., rows, cols] tensor whose rows are contiguous; an axis of one element takes any."""
    rows, cols = t.shape[-2:]
    if cols > 1 and t.stride(-1) != 1:
        raise ValueError(f"the last axis of {name} must be contiguous")
    row = t.stride(-2) if rows > 1 else max(cols, 1)
    if row < cols:
        raise ValueError(f"the rows of {name} overlap")
    if t.dim() == 2 or t.shape[0] <= 1:
        return row, 0
    return row, t.stride(0)


def _parameter_stride(name: str, t: torch.Tensor) -> int:
    """Stride between the workers' parts of a parameter whose own part is contiguous (t has a worker axis)."""
    part = t[0] if t.dim() and t.shape[0] else t
    if not part.is_contiguous():
        raise ValueError(f"each worker's part of {name} must be contiguous")
    return t.stride(0) if t.shape[0] > 1 else 0


# ------------------------------------------------------------------------------------------------------------ the loss
class _LcePlan(NamedTuple):
    desc: object
    tokens: object                   # layouts
    loss: object
    hidden: object
    weight: object
    sizes: Tuple[int, int]           # bytes of workspace, forward and backward
    workspace: Tuple[object, object]


def _lce_plan(hidden, weight, targets, ignore_index, reduction, dweight=None) -> _LcePlan:
    at = weight.data_ptr() & 15
    key = ("lce", hidden.dtype, hidden.shape, hidden.stride(), weight.dtype, weight.shape, weight.stride(), at, targets.dtype, targets.shape,
           ignore_index, reduction) + (() if dweight is None else (dweight.dtype, dweight.shape, dweight.stride()))
    plan = _plans.get(key)
    if plan is not None:
        return plan
    if reduction not in _REDUCTION:
        raise ValueError(f"reduction must be one of {sorted(_REDUCTION)}")
    if hidden.dim() not in (2, 3):
        raise ValueError("hidden must be a tensor [n, tokens, cols] or [tokens, cols]")
    lead = tuple(hidden.shape[:-2])
    tokens, cols = hidden.shape[-2:]
    _check("hidden", hidden, None, tuple(hidden.shape))
    if weight.dim() != hidden.dim():
        raise ValueError("weight must be [n, vocab, cols] with hidden [n, tokens, cols], or [vocab, cols] with [tokens, cols]")
    vocab = weight.shape[-2]
    _check("weight", weight, hidden, lead + (vocab, cols))
    if targets.dtype != torch.int64 or tuple(targets.shape) != lead + (tokens,):
        raise ValueError(f"targets must be int64 of shape {lead + (tokens,)}, not {targets.dtype} of {tuple(targets.shape)}")
    d = rps_lce_desc(dtype=_DTYPE[hidden.dtype], reduction=_REDUCTION[reduction], n=lead[0] if lead else 1, tokens=tokens,
                     vocab=vocab, cols=cols, ignore_index=ignore_index)
    d.hidden_row, d.hidden_worker = _matrix_strides("hidden", hidden)
    d.weight_row, d.weight_worker = _matrix_strides("weight", weight)
    if dweight is not None:
        _check("dweight", dweight, hidden, tuple(weight.shape))
        d.dweight_row, d.dweight_worker = _matrix_strides("dweight", dweight)
    else:
        d.dweight_row, d.dweight_worker = cols, vocab * cols
    sizes = []
    for backward in (0, 1):
        size = ctypes.c_size_t()
        _call("rps_lce_workspace", hidden.get_device(), ctypes.byref(d), at, backward, ctypes.byref(size))
        sizes.append(size.value)
    each = _dense_layout(lead + (tokens,))
    return _keep(key, _LcePlan(ctypes.byref(d), each, each if reduction == "none" else _dense_layout(lead), _dense_layout(hidden.shape),
                               _dense_layout(weight.shape), tuple(sizes), tuple(_dense_layout((size,)) for size in sizes)))


def linear_cross_entropy_forward(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, *,
                                 ignore_index: int = -100, reduction: str = "mean") -> Tuple[torch.Tensor, torch.Tensor]:
    """(loss, lse) of ``hidden @ weight.T`` against ``targets`` (``rps_lce_forward``).

    hidden ``[n, tokens, cols]``, weight ``[n, vocab, cols]``, targets int64 ``[n, tokens]`` (all without ``n`` for a single
    worker).  loss is float32: one value for each worker ("mean" over its tokens that are not ignored, "sum") or each token
    ("none"); lse, float32 ``[n, tokens]``, is what the backward pass wants.  Ignored tokens have loss and lse 0."""
    device = _device_of(hidden=hidden, weight=weight, targets=targets)
    plan = _lce_plan(hidden, weight, targets, ignore_index, reduction)
    targets = targets.contiguous()
    where = hidden.device
    loss, lse = _new(plan.loss, torch.float32, where), _new(plan.tokens, torch.float32, where)
    ws = _new(plan.workspace[0], torch.uint8, where)
    _call("rps_lce_forward", device, plan.desc, hidden.data_ptr(), weight.data_ptr(), targets.data_ptr(), loss.data_ptr(), lse.data_ptr(),
          ws.data_ptr(), plan.sizes[0], _stream(device))
    return loss, lse


def linear_cross_entropy_backward(dloss: torch.Tensor, hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor,
                                  lse: torch.Tensor, *, ignore_index: int = -100, reduction: str = "mean",
                                  dweight: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(dhidden, dweight) for the gradient ``dloss`` (float32, shaped as the loss) of the forward call with the same
    arguments (``rps_lce_backward``).  ``dweight``, if given, is written (not added to) and may be strided, a view into
    the rows of a larger array for instance."""
    device = _device_of(hidden=hidden, weight=weight, targets=targets, dloss=dloss, lse=lse)
    if dweight is not None:
        _device_of(hidden=hidden, dweight=dweight)
    plan = _lce_plan(hidden, weight, targets, ignore_index, reduction, dweight)
    targets = targets.contiguous()
    for name, t, shape in (("dloss", dloss, plan.loss[0]), ("lse", lse, plan.tokens[0])):
        if t.dtype != torch.float32 or t.shape != shape:
            raise ValueError(f"{name} must be a float32 tensor of shape {shape}")
        _dense(name, t)
    where = hidden.device
    if dweight is None:
        dweight = _new(plan.weight, weight.dtype, where)
    dhidden = _new(plan.hidden, hidden.dtype, where)
    ws = _new(plan.workspace[1], torch.uint8, where)
    _call("rps_lce_backward", device, plan.desc, hidden.data_ptr(), weight.data_ptr(), targets.data_ptr(), lse.data_ptr(), dloss.data_ptr(),
          dhidden.data_ptr(), dweight.data_ptr(), ws.data_ptr(), plan.sizes[1], _stream(device))
    return dhidden, dweight


class _LinearCrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, weight, targets, ignore_index, reduction):
        loss, lse = linear_cross_entropy_forward(hidden, weight, targets, ignore_index=ignore_index, reduction=reduction)
        ctx.save_for_backward(hidden, weight, targets, lse)
        ctx.settings = {"ignore_index": ignore_index, "reduction": reduction}
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        dhidden, dweight = linear_cross_entropy_backward(dloss.float().contiguous(), *ctx.saved_tensors, **ctx.settings)
        return dhidden, dweight, None, None, None


def linear_cross_entropy(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, *, ignore_index: int = -100,
                         reduction: str = "mean") -> torch.Tensor:
    """Differentiable ``linear_cross_entropy_forward``: the loss alone."""
    return _LinearCrossEntropy.apply(hidden, weight, targets, ignore_index, reduction)


# ------------------------------------------------------------------------------------------------------ 8-bit activations
class PackedActivation(NamedTuple):
    """Activations ``[..., columns]`` in 8 bits: int8 codes ``[..., columns rounded up to 16]`` and a float32 scale for each
    128 columns, ``[..., groups]``; ``dtype`` is the type that they are read back in."""

    codes: torch.Tensor
    scales: torch.Tensor
    columns: int
    dtype: torch.dtype


def _packed_layout(shape):
    """Layouts of the codes and the scales of a tensor of this shape."""
    lead, cols = tuple(shape[:-1]), shape[-1]
    return _dense_layout(lead + (-(-cols // 16) * 16,)), _dense_layout(lead + (-(-cols // GROUP),))


def packed_like(shape: Tuple[int, ...], dtype: torch.dtype, device: torch.device) -> PackedActivation:
    """Room for the packed form of a tensor of this shape (the codes behind the last column are written by pack calls)."""
    codes, scales = _packed_layout(shape)
    return PackedActivation(_new(codes, torch.int8, device), _new(scales, torch.float32, device), shape[-1], dtype)


def _packed_for(name: str, p: PackedActivation):
    """Checks ``p`` and gives the layout of the tensor that it stands for."""
    if not isinstance(p, PackedActivation):
        raise ValueError(f"{name} must be a PackedActivation")
    c, s = p.codes, p.scales
    key = ("packed", c.dtype, c.shape, c.stride(), s.dtype, s.shape, s.stride(), p.columns, p.dtype)
    layout = _plans.get(key)
    if layout is not None:
        return layout
    if c.dtype != torch.int8 or s.dtype != torch.float32:
        raise ValueError(f"{name}: codes must be int8 and scales float32")
    if p.dtype not in _DTYPE:
        raise ValueError(f"{name}: dtype must be float32 or bfloat16")
    if p.columns < 1 or c.dim() < 1 or c.shape[-1] != -(-p.columns // 16) * 16 or tuple(s.shape) != tuple(c.shape[:-1]) + (-(-p.columns // GROUP),):
        raise ValueError(f"{name}: codes {tuple(c.shape)} and scales {tuple(s.shape)} do not fit {p.columns} columns")
    _dense(f"{name}.codes", c)
    _dense(f"{name}.scales", s)
    return _keep(key, _dense_layout(tuple(c.shape[:-1]) + (p.columns,)))


def pack_activation(x: torch.Tensor) -> PackedActivation:
    """``x`` in 8 bits (``rps_pack``).  x is ``[..., columns]`` and contiguous, or a matrix with contiguous rows."""
    device = _device_of(x=x)
    key = ("pack", x.dtype, x.shape, x.stride())
    plan = _plans.get(key)
    if plan is None:
        if x.dim() < 1 or x.shape[-1] < 1:
            raise ValueError("x must be a tensor [..., columns] with at least one column")
        _check("x", x, None, tuple(x.shape))
        row = _matrix_strides("x", x)[0] if x.dim() == 2 else x.shape[-1]
        if x.dim() != 2:
            _dense("x", x)
        plan = _keep(key, (_DTYPE[x.dtype], x.numel() // x.shape[-1], x.shape[-1], row) + _packed_layout(x.shape))
    dtype, rows, cols, row, codes, scales = plan
    where = x.device
    codes, scales = _new(codes, torch.int8, where), _new(scales, torch.float32, where)
    _call("rps_pack", device, dtype, rows, cols, x.data_ptr(), row, codes.data_ptr(), scales.data_ptr(), _stream(device))
    return PackedActivation(codes, scales, cols, x.dtype)


def unpack_activation(packed: PackedActivation) -> torch.Tensor:
    """The values that ``packed`` stands for, in its dtype (``rps_unpack``)."""
    layout = _packed_for("packed", packed)
    codes, scales, cols, dtype = packed
    device = _device_of(codes=codes, scales=scales)
    out = _new(layout, dtype, codes.device)
    _call("rps_unpack", device, _DTYPE[dtype], out.numel() // cols, cols, codes.data_ptr(), scales.data_ptr(), out.data_ptr(), cols,
          _stream(device))
    return out


def packed_weight_grad(dy: torch.Tensor, packed: PackedActivation, *, dweight: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``dy.mT @ x`` for the values x that ``packed`` stands for (``rps_packed_wgrad``): the weight gradient
    ``[n, outs, columns]`` of ``y = x @ weight.mT`` out of dy ``[n, tokens, outs]``.  ``dweight`` as in
    ``linear_cross_entropy_backward``."""
    shape = _packed_for("packed", packed)[0]
    device = _device_of(dy=dy, codes=packed.codes, scales=packed.scales)
    if dweight is not None:
        _device_of(dy=dy, dweight=dweight)
    at = dy.data_ptr() & 15
    key = ("wgrad", dy.dtype, dy.shape, dy.stride(), at, shape, packed.dtype) + (() if dweight is None else (dweight.dtype, dweight.shape, dweight.stride()))
    plan = _plans.get(key)
    if plan is None:
        if dy.dim() not in (2, 3) or dy.shape[-1] < 1:
            raise ValueError("dy must be a tensor [n, tokens, outs] or [tokens, outs]")
        _check("dy", dy, None, tuple(dy.shape))
        lead, (tokens, outs), cols = tuple(dy.shape[:-2]), dy.shape[-2:], packed.columns
        if shape != lead + (tokens, cols):
            raise ValueError(f"packed must stand for a tensor {lead + (tokens, cols)}, not {shape}")
        if packed.dtype != dy.dtype:
            raise ValueError("dy and packed must have one type")
        d = rps_wgrad_desc(dtype=_DTYPE[dy.dtype], n=lead[0] if lead else 1, tokens=tokens, outs=outs, cols=cols)
        d.dy_row, d.dy_worker = _matrix_strides("dy", dy)
        d.dweight_row, d.dweight_worker = cols, outs * cols
        if dweight is not None:
            _check("dweight", dweight, dy, lead + (outs, cols))
            d.dweight_row, d.dweight_worker = _matrix_strides("dweight", dweight)
        size = ctypes.c_size_t()
        _call("rps_wgrad_workspace", device, ctypes.byref(d), at, ctypes.byref(size))
        plan = _keep(key, (ctypes.byref(d), _dense_layout(lead + (outs, cols)), _dense_layout((size.value,)), size.value))
    desc, out_layout, ws_layout, size = plan
    if dweight is None:
        dweight = _new(out_layout, dy.dtype, dy.device)
    ws = _new(ws_layout, torch.uint8, dy.device)
    _call("rps_packed_wgrad", device, desc, dy.data_ptr(), packed.codes.data_ptr(), packed.scales.data_ptr(), dweight.data_ptr(), ws.data_ptr(),
          size, _stream(device))
    return dweight


class _Linear8bit(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight):
        packed = pack_activation(x.contiguous())
        ctx.save_for_backward(packed.codes, packed.scales, weight)
        ctx.kept = packed.columns, packed.dtype
        return torch.matmul(x, weight.mT)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        codes, scales, weight = ctx.saved_tensors
        dy = dy.contiguous()
        return torch.matmul(dy, weight), packed_weight_grad(dy, PackedActivation(codes, scales, *ctx.kept))


def linear_8bit(x: torch.Tensor, weight: torch.Tensor) -> torch.Tensor:
    """``x @ weight.mT`` with the input kept in 8 bits for the weight gradient: x ``[n, tokens, cols]``, weight ``[n, outs, cols]``,
    or both without ``n``.  The two plain products are PyTorch's."""
    if x.dim() != weight.dim() or x.dim() not in (2, 3):
        raise ValueError("x must be [n, tokens, cols] with weight [n, outs, cols], or [tokens, cols] with [outs, cols]")
    _device_of(x=x, weight=weight)
    _check("x", x, None, tuple(x.shape))
    _check("weight", weight, x, tuple(x.shape[:-2]) + (weight.shape[-2], x.shape[-1]))
    return _Linear8bit.apply(x, weight)


# ------------------------------------------------------------------------------------------------- norms around a block
class GatedResidualNormKept(NamedTuple):
    """What ``gated_residual_norm_backward`` reads of the forward pass: f and h (tensors, or both packed) and the
    reciprocal root mean squares of their rows, float32 ``[2, n, tokens]``."""

    f: object
    h: object
    r: torch.Tensor
    eps: float

    @property
    def r_f(self) -> torch.Tensor:
        return self.r[0]

    @property
    def r_h(self) -> torch.Tensor:
        return self.r[1]


def _norm_plan(x, gate, post, pre, scale, eps):
    """(description, bytes between r_f and r_h, layout of both, bytes of workspace of the backward pass, its layout)"""
    key = ("norm", x.dtype, x.shape, x.stride(), gate.dtype, gate.shape, gate.stride(), post.dtype, post.shape, post.stride(), pre.dtype,
           pre.shape, pre.stride(), scale, eps)
    plan = _plans.get(key)
    if plan is not None:
        return plan
    if x.dim() not in (2, 3):
        raise ValueError("x must be a tensor [n, tokens, cols] or [tokens, cols]")
    _check("x", x, None, tuple(x.shape))
    _dense("x", x)
    lead, (tokens, cols) = tuple(x.shape[:-2]), x.shape[-2:]
    if gate.dim() != x.dim():
        raise ValueError("gate must be [n, gates, cols] with x [n, tokens, cols], or [gates, cols] with [tokens, cols]")
    gates = gate.shape[-2]
    _check("gate", gate, x, lead + (gates, cols))
    _check("post", post, x, lead + (cols,))
    _check("pre", pre, x, lead + (cols,))
    n = lead[0] if lead else 1
    d = rps_norm_desc(dtype=_DTYPE[x.dtype], n=n, tokens=tokens, cols=cols, gates=gates, scale=scale, eps=eps)
    d.post_worker, d.pre_worker, d.gate_worker = (_parameter_stride(name, t if lead else t[None])
                                                  for name, t in (("post", post), ("pre", pre), ("gate", gate)))
    size = ctypes.c_size_t()
    _call("rps_norm_workspace", x.get_device(), ctypes.byref(d), ctypes.byref(size))
    return _keep(key, (ctypes.byref(d), 4 * n * tokens, _dense_layout((2,) + lead + (tokens,)), size.value, _dense_layout((size.value,))))


def _same(name: str, t: torch.Tensor, like: torch.Tensor) -> None:
    """t is laid out as ``like``, which is contiguous."""
    if t.dtype != like.dtype or t.shape != like.shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {like.dtype} tensor of shape {tuple(like.shape)}")


def gated_residual_norm_forward(x: torch.Tensor, f: torch.Tensor, gate: torch.Tensor, post: torch.Tensor, pre: torch.Tensor, *,
                                scale: float = 1.0, eps: float = 1e-6, keep: str = "values"):
    """(h, y, kept) with ``h = x + scale * gate * norm(f) * post`` and ``y = norm(h) * pre``, norm being division by the
    root mean square of a row (``rps_norm_forward``).

    x, f ``[n, tokens, cols]``; post, pre ``[n, cols]``; gate ``[n, gates, cols]``, gates a divisor of tokens (consecutive tokens
    share a row: 1 for a gate of each channel, tokens for one of each token); all without ``n`` for a single worker.
    keep: "values" (kept holds f and h themselves: a bfloat16 h as it is rounded), "int8" (8-bit copies, written along the way).
    scale and eps are numbers and get no gradient."""
    if keep not in ("values", "int8"):
        raise ValueError('keep must be "values" or "int8"')
    device = _device_of(x=x, f=f, gate=gate, post=post, pre=pre)
    scale, eps = float(scale), float(eps)  # a number held in a tensor too: plans are kept by values, never by what holds one
    desc, between, r_layout, _, _ = _norm_plan(x, gate, post, pre, scale, eps)
    _same("f", f, x)
    h, y = torch.empty_like(x), torch.empty_like(x)
    r = _new(r_layout, torch.float32, x.device)
    r_f = r.data_ptr()
    if keep == "int8":
        kept_f, kept_h = packed_like(x.shape, x.dtype, x.device), packed_like(x.shape, x.dtype, x.device)
        packed = kept_f.codes.data_ptr(), kept_f.scales.data_ptr(), kept_h.codes.data_ptr(), kept_h.scales.data_ptr()
    else:
        kept_f, kept_h = f, h
        packed = None, None, None, None
    _call("rps_norm_forward", device, desc, x.data_ptr(), f.data_ptr(), gate.data_ptr(), post.data_ptr(), pre.data_ptr(), h.data_ptr(),
          y.data_ptr(), r_f, r_f + between, *packed, _stream(device))
    return h, y, GatedResidualNormKept(kept_f, kept_h, r, eps)


def gated_residual_norm_backward(dh: Optional[torch.Tensor], dy: torch.Tensor, kept: GatedResidualNormKept, gate: torch.Tensor,
                                 post: torch.Tensor, pre: torch.Tensor, *, scale: float = 1.0):
    """(dx, df, dgate, dpost, dpre) for the gradients dh (None: none reaches h but through y) and dy of the forward call's h
    and y (``rps_norm_backward``)."""
    device = _device_of(dy=dy, gate=gate, post=post, pre=pre, r=kept.r)
    desc, between, r_layout, size, ws_layout = _norm_plan(dy, gate, post, pre, float(scale), float(kept.eps))
    if dh is not None:
        _device_of(dy=dy, dh=dh)
        _same("dh", dh, dy)
    if isinstance(kept.f, PackedActivation):
        _device_of(dy=dy, f_codes=kept.f.codes, f_scales=kept.f.scales, h_codes=kept.h.codes, h_scales=kept.h.scales)
        for name, p in (("kept.f", kept.f), ("kept.h", kept.h)):
            if _packed_for(name, p)[0] != dy.shape or p.dtype != dy.dtype:
                raise ValueError(f"{name} does not go with dy")
        f, f_scales, h, h_scales = (t.data_ptr() for t in (kept.f.codes, kept.f.scales, kept.h.codes, kept.h.scales))
    else:
        _device_of(dy=dy, f=kept.f, h=kept.h)
        _same("kept.f", kept.f, dy)
        _same("kept.h", kept.h, dy)
        f, f_scales, h, h_scales = kept.f.data_ptr(), None, kept.h.data_ptr(), None
    r = kept.r
    if r.dtype != torch.float32 or r.shape != r_layout[0] or not r.is_contiguous():
        raise ValueError(f"kept.r must be a contiguous float32 tensor of shape {r_layout[0]}")
    dx, df = torch.empty_like(dy), torch.empty_like(dy)
    dgate, dpost, dpre = (torch.empty_like(t, memory_format=torch.contiguous_format) for t in (gate, post, pre))
    ws = _new(ws_layout, torch.uint8, dy.device)
    _call("rps_norm_backward", device, desc, None if dh is None else dh.data_ptr(), dy.data_ptr(), f, f_scales, h, h_scales, r.data_ptr(),
          r.data_ptr() + between, gate.data_ptr(), post.data_ptr(), pre.data_ptr(), dx.data_ptr(), df.data_ptr(), dgate.data_ptr(),
          dpost.data_ptr(), dpre.data_ptr(), ws.data_ptr(), size, _stream(device))
    return dx, df, dgate, dpost, dpre


class _GatedResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, f, gate, post, pre, scale, eps, keep):
        h, y, kept = gated_residual_norm_forward(x, f, gate, post, pre, scale=scale, eps=eps, keep=keep)
        ctx.set_materialize_grads(False)
        ctx.settings = scale, eps, keep
        if keep == "int8":
            ctx.columns = kept.f.columns, kept.f.dtype
            ctx.save_for_backward(gate, post, pre, kept.r, kept.f.codes, kept.f.scales, kept.h.codes, kept.h.scales)
        else:
            ctx.save_for_backward(gate, post, pre, kept.r, f, h)
        return h, y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dh, dy):
        scale, eps, keep = ctx.settings
        gate, post, pre, r, *rest = ctx.saved_tensors
        if keep == "int8":
            f, h = (PackedActivation(c, s, *ctx.columns) for c, s in (rest[:2], rest[2:]))
        else:
            f, h = rest
        if dy is None:  # y was not used
            dy = torch.zeros(r.shape[1:] + (post.shape[-1],), dtype=post.dtype, device=post.device)
        grads = gated_residual_norm_backward(None if dh is None else dh.contiguous(), dy.contiguous(),
                                             GatedResidualNormKept(f, h, r, eps), gate, post, pre, scale=scale)
        return grads + (None, None, None)


def gated_residual_norm(x: torch.Tensor, f: torch.Tensor, gate: torch.Tensor, post: torch.Tensor, pre: torch.Tensor, *,
                        scale: float = 1.0, eps: float = 1e-6, keep: str = "values") -> Tuple[torch.Tensor, torch.Tensor]:
    """Differentiable ``gated_residual_norm_forward``: (h, y)."""
    for name, v in (("scale", scale), ("eps", eps)):
        if isinstance(v, torch.Tensor) and v.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{name} gets no gradient: a learned factor belongs into gate or post")
    return _GatedResidualNorm.apply(x, f, gate, post, pre, float(scale), float(eps), keep)
