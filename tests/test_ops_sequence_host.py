"""Host-side checks of the operators on sequences: what needs no GPU refuses bad arguments with a status and a reason."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_1810_07766_b200 import build, ops

    build.build()
    return ops._library()


def embed_desc(**changes):
    from paper_1810_07766_b200 import ops

    d = ops.rps_embed_desc(dtype=1, n=2, tokens=5, vocab=7, cols=8, ignore_index=-100, weight_row=8, weight_worker=56, dweight_row=8, dweight_worker=56, scale=1.0)
    for k, v in changes.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change", [{"dtype": 2}, {"n": 0}, {"n": 65}, {"accumulate": 2}, {"accumulate": -1}, {"reserved": 1}, {"tokens": -1}, {"tokens": 1 << 24},
                                    {"vocab": 0}, {"vocab": 1 << 30}, {"cols": 0}, {"cols": 1 << 24}, {"scale": float("inf")}, {"scale": float("nan")}])
def test_embedding_descriptions_are_refused(lib, change):
    size, one = ctypes.c_size_t(), 256
    assert lib.rps_embed_workspace(ctypes.byref(embed_desc()), ctypes.byref(size)) == 0 and size.value > 0
    assert lib.rps_ops_last_error() == b""
    d = ctypes.byref(embed_desc(**change))
    assert lib.rps_embed_workspace(d, ctypes.byref(size)) == -1 and lib.rps_ops_last_error()
    assert lib.rps_embed_forward(d, one, one, one, None) == -1
    assert lib.rps_embed_backward(d, one, one, one, one, 1 << 20, None) == -1
    assert lib.rps_embed_workspace(None, ctypes.byref(size)) == -1
    assert lib.rps_embed_workspace(ctypes.byref(embed_desc()), None) == -1


def test_embedding_arrays_are_refused(lib):
    size, one = ctypes.c_size_t(), 256
    lib.rps_embed_workspace(ctypes.byref(embed_desc()), ctypes.byref(size))
    for at in range(3):
        args = [one] * 3
        args[at] = None
        assert lib.rps_embed_forward(ctypes.byref(embed_desc()), *args, None) == -1
        assert lib.rps_embed_backward(ctypes.byref(embed_desc()), *args, one, size.value, None) == -1
    for change in ({"weight_row": 7}, {"weight_worker": -1}):
        assert lib.rps_embed_forward(ctypes.byref(embed_desc(**change)), one, one, one, None) == -1
    for change in ({"dweight_row": 7}, {"dweight_worker": 55}, {"dweight_worker": 0}, {"dweight_row": 15, "dweight_worker": 8}, {"dweight_row": 1 << 31}):
        assert lib.rps_embed_backward(ctypes.byref(embed_desc(**change)), one, one, one, one, size.value, None) == -1
        assert b"dweight" in lib.rps_ops_last_error()
    for ws, have in ((one, size.value - 1), (None, size.value), (264, size.value)):
        assert lib.rps_embed_backward(ctypes.byref(embed_desc()), one, one, one, ws, have, None) == -1
        assert b"workspace" in lib.rps_ops_last_error()
    assert lib.rps_embed_forward(ctypes.byref(embed_desc(tokens=0)), None, None, None, None) == 0   # nothing to do


def test_embedding_refuses_cpu_tensors():
    from paper_1810_07766_b200 import ops

    y, w = torch.zeros(4, dtype=torch.int64), torch.zeros(6, 8)
    with pytest.raises(ValueError, match="CUDA"):
        ops.embedding(y, w)
    with pytest.raises(ValueError, match="CUDA"):
        ops.embedding_backward(w[:4], y, 6)
