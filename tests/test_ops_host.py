"""Host-side checks of the training operators: every symbol of include/rps_ops.h is exported, and what needs no GPU refuses bad
arguments with a status and a reason."""
import ctypes
import os
import re

import pytest
import torch

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "rps_ops.h")


@pytest.fixture(scope="module")
def lib():
    from paper_1810_07766_b200 import build, ops

    build.build()
    return ops._library()


def test_header_symbols_are_exported(lib):
    from paper_1810_07766_b200 import ops

    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(rps_[a-z_0-9]+)\s*\(", text)))
    assert sorted(ops.SYMBOLS) == names
    for name in names:
        assert getattr(lib, name) is not None


def lce_desc(**changes):
    from paper_1810_07766_b200 import ops

    d = ops.rps_lce_desc(dtype=1, reduction=2, n=2, tokens=5, vocab=7, cols=8, ignore_index=-100, hidden_row=8, hidden_worker=40,
                         weight_row=8, weight_worker=56, dweight_row=8, dweight_worker=56)
    for k, v in changes.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change", [{"dtype": 2}, {"dtype": -1}, {"reduction": 3}, {"reduction": -1}, {"n": 0}, {"n": 65}, {"tokens": -1},
                                    {"tokens": 1 << 24}, {"vocab": 0}, {"vocab": 1 << 30}, {"cols": 0}, {"hidden_row": 7},
                                    {"weight_row": 7}, {"hidden_worker": -1}, {"weight_worker": -1}])
def test_loss_descriptions_are_refused(lib, change):
    size = ctypes.c_size_t()
    for backward in (0, 1):
        assert lib.rps_lce_workspace(ctypes.byref(lce_desc()), None, backward, ctypes.byref(size)) == 0 and size.value > 0
        assert lib.rps_ops_last_error() == b""
        assert lib.rps_lce_workspace(ctypes.byref(lce_desc(**change)), None, backward, ctypes.byref(size)) == -1
        assert lib.rps_ops_last_error()
    assert lib.rps_lce_workspace(None, None, 0, ctypes.byref(size)) == -1
    assert lib.rps_lce_workspace(ctypes.byref(lce_desc()), None, 0, None) == -1


def test_loss_arrays_and_workspaces_are_refused(lib):
    d, one = lce_desc(), 256
    size = ctypes.c_size_t()
    lib.rps_lce_workspace(ctypes.byref(d), one, 0, ctypes.byref(size))
    assert lib.rps_lce_forward(ctypes.byref(d), None, one, one, one, one, one, size.value, None) == -1
    assert lib.rps_lce_forward(ctypes.byref(d), one, None, one, one, one, one, size.value, None) == -1
    assert lib.rps_lce_forward(ctypes.byref(d), one, one, one, None, one, one, size.value, None) == -1
    assert lib.rps_lce_forward(ctypes.byref(d), one, one, one, one, one, one, size.value - 1, None) == -1
    assert b"workspace" in lib.rps_ops_last_error()
    assert lib.rps_lce_forward(ctypes.byref(d), one, one, one, one, one, None, size.value, None) == -1
    assert lib.rps_lce_forward(ctypes.byref(d), one, one, one, one, one, 264, size.value, None) == -1
    lib.rps_lce_workspace(ctypes.byref(d), one, 1, ctypes.byref(size))
    assert lib.rps_lce_backward(ctypes.byref(d), one, one, one, one, one, one, None, one, size.value, None) == -1
    # the workers' gradients must not overlap, and a row of them holds all columns
    for change in ({"dweight_row": 7}, {"dweight_worker": 55}, {"dweight_worker": 0}, {"dweight_row": 15, "dweight_worker": 8}):
        assert lib.rps_lce_backward(ctypes.byref(lce_desc(**change)), one, one, one, one, one, one, one, one, size.value, None) == -1
        assert b"dweight" in lib.rps_ops_last_error()


def test_norm_descriptions_are_refused(lib):
    from paper_1810_07766_b200 import ops

    def desc(**changes):
        d = ops.rps_norm_desc(dtype=0, n=2, tokens=6, cols=10, gates=3, post_worker=10, pre_worker=10, gate_worker=30, scale=1.0, eps=1e-6)
        for k, v in changes.items():
            setattr(d, k, v)
        return d

    size = ctypes.c_size_t()
    assert lib.rps_norm_workspace(ctypes.byref(desc()), ctypes.byref(size)) == 0 and size.value > 0
    for change in ({"dtype": 5}, {"n": 0}, {"n": 65}, {"tokens": -1}, {"tokens": 7}, {"gates": 0}, {"gates": 4}, {"gates": 12}, {"cols": 0},
                   {"post_worker": -1}, {"pre_worker": -1}, {"gate_worker": -1}, {"scale": float("inf")}, {"scale": float("nan")},
                   {"eps": -1.0}, {"eps": float("nan")}, {"tokens": 0, "gates": 2}, {"tokens": 1 << 31, "gates": 1}):
        assert lib.rps_norm_workspace(ctypes.byref(desc(**change)), ctypes.byref(size)) == -1, change
        assert lib.rps_ops_last_error()
    assert lib.rps_norm_workspace(ctypes.byref(desc(cols=ops.MAX_NORM_COLS + 1)), ctypes.byref(size)) == -5
    one = 256
    args = [one] * 14
    for at, bad in ((0, None), (1, None), (7, None), (9, None), (12, None), (9, 264)):
        a = list(args)
        a[at] = bad
        assert lib.rps_norm_forward(ctypes.byref(desc()), *a) == -1, at
    back = [one] * 17 + [size.value, None]
    for at, bad in ((1, None), (2, None), (3, None), (7, None), (12, None), (14, None), (16, None), (3, 264)):
        a = list(back)
        a[at] = bad
        assert lib.rps_norm_backward(ctypes.byref(desc()), *a) == -1, at


def test_pack_and_wgrad_arguments_are_refused(lib):
    from paper_1810_07766_b200 import ops

    one = 256
    assert [lib.rps_pack_pitch(c) for c in (1, 16, 17, 1000)] == [16, 16, 32, 1008]
    for call in (lambda *a: lib.rps_pack(a[0], a[1], a[2], a[3], a[4], a[5], a[6], None),
                 lambda *a: lib.rps_unpack(a[0], a[1], a[2], a[5], a[6], a[3], a[4], None)):
        for bad in ((2, 3, 10, one, 10, one, one), (0, -1, 10, one, 10, one, one), (0, 3, 0, one, 10, one, one), (0, 3, 10, one, 9, one, one),
                    (0, 3, 10, None, 10, one, one), (0, 3, 10, one, 10, None, one), (0, 3, 10, one, 10, one, None),
                    (0, 3, 10, one, 10, one + 8, one), (0, 3, 10, one, 10, one, one + 4), (0, 1 << 31, 10, one, 10, one, one)):
            assert call(*bad) == -1, bad
        assert call(0, 0, 10, None, 10, None, None) == 0   # nothing to do

    def desc(**changes):
        d = ops.rps_wgrad_desc(dtype=1, n=2, tokens=5, outs=8, cols=10, dy_row=8, dy_worker=40, dweight_row=10, dweight_worker=80)
        for k, v in changes.items():
            setattr(d, k, v)
        return d

    size = ctypes.c_size_t()
    assert lib.rps_wgrad_workspace(ctypes.byref(desc()), None, ctypes.byref(size)) == 0 and size.value > 0
    for change in ({"dtype": 2}, {"n": 0}, {"tokens": -1}, {"outs": 0}, {"cols": 0}, {"dy_row": 7}, {"dy_worker": -1}, {"dweight_row": 9},
                   {"dweight_worker": 79}, {"dweight_row": 1 << 31, "dweight_worker": 1 << 40}, {"wait_limit_ms": -1}, {"withhold_copies": 2}):
        assert lib.rps_wgrad_workspace(ctypes.byref(desc(**change)), None, ctypes.byref(size)) == -1, change
    assert lib.rps_packed_wgrad(ctypes.byref(desc()), one, one, one, None, one, size.value, None) == -1
    assert lib.rps_packed_wgrad(ctypes.byref(desc()), one, one, one, one, one, size.value - 1, None) == -1
    assert lib.rps_packed_wgrad(ctypes.byref(desc()), one, one + 8, one, one, one, size.value, None) == -1


def test_cpu_tensors_are_refused():
    from paper_1810_07766_b200 import ops

    h, w, y = torch.zeros(4, 8), torch.zeros(6, 8), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="CUDA"):
        ops.linear_cross_entropy(h, w, y)
    with pytest.raises(ValueError, match="CUDA"):
        ops.gated_residual_norm(h, h, h[:1], h[0], h[0])
    with pytest.raises(ValueError, match="CUDA"):
        ops.pack_activation(h)
    with pytest.raises(ValueError, match="CUDA"):
        ops.packed_weight_grad(h, ops.packed_like((4, 8), torch.float32, torch.device("cpu")))
