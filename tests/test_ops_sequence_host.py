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


def attention_desc(**changes):
    from paper_1810_07766_b200 import ops

    d = ops.rps_linear_attention_desc(dtype=1, n=2, heads=3, sequences=4, tokens=5, key_cols=8, value_cols=16, scale=1.0)
    for k, v in changes.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change", [{"dtype": 2}, {"n": 0}, {"n": 65}, {"heads": 0}, {"heads": 65536}, {"reserved": 1}, {"sequences": -1}, {"sequences": 1 << 28},
                                    {"sequences": 1 << 27}, {"tokens": -1}, {"tokens": 1 << 31}, {"key_cols": 0}, {"value_cols": 0}, {"scale": float("inf")},
                                    {"scale": float("nan")}, {"q": (-1, 0, 0, 0)}, {"k": (0, -1, 0, 0)}, {"v": (0, 0, -1, 0)}, {"dout": (0, 0, 0, -1)}])
def test_attention_descriptions_are_refused(lib, change):
    from paper_1810_07766_b200 import ops

    size, one = ctypes.c_size_t(), 256
    change = {k: ops.rps_axis_strides(*v) if isinstance(v, tuple) else v for k, v in change.items()}
    d = ctypes.byref(attention_desc(**change))
    for backward in (0, 1):
        assert lib.rps_linear_attention_workspace(ctypes.byref(attention_desc()), backward, ctypes.byref(size)) == 0
        assert lib.rps_linear_attention_workspace(d, backward, ctypes.byref(size)) == -1 and lib.rps_ops_last_error()
    assert lib.rps_linear_attention_forward(d, *[one] * 9, 1 << 20, None) == -1
    assert lib.rps_linear_attention_backward(d, *[one] * 13, 1 << 20, None) == -1
    assert lib.rps_linear_attention_step(d, *[one] * 7, None) == -1


def test_attention_arrays_are_refused(lib):
    from paper_1810_07766_b200 import ops

    size, one = ctypes.c_size_t(), 256
    assert lib.rps_linear_attention_workspace(None, 0, ctypes.byref(size)) == -1
    assert lib.rps_linear_attention_workspace(ctypes.byref(attention_desc()), 0, None) == -1
    for cols in ({"key_cols": ops.MAX_HEAD_COLS + 1}, {"value_cols": ops.MAX_HEAD_COLS + 1}):
        assert lib.rps_linear_attention_workspace(ctypes.byref(attention_desc(**cols)), 0, ctypes.byref(size)) == -5
    d = ctypes.byref(attention_desc())
    for at in (0, 1, 2, 3, 6):
        args = [one] * 9
        args[at] = None
        assert lib.rps_linear_attention_forward(d, *args, 0, None) == -1
    for at in (0, 2, 3, 4, 5, 8, 9, 10):
        args = [one] * 13
        args[at] = None
        assert lib.rps_linear_attention_backward(d, *args, 0, None) == -1
    single = ctypes.byref(attention_desc(tokens=1))
    assert lib.rps_linear_attention_step(d, *[one] * 7, None) == -1   # 5 tokens
    for at in range(7):
        args = [one] * 7
        args[at] = None
        assert lib.rps_linear_attention_step(single, *args, None) == -1
    # a long sequence of few heads goes through in segments, which want a workspace
    long = attention_desc(n=1, heads=1, sequences=1, tokens=100_000)
    assert lib.rps_linear_attention_workspace(ctypes.byref(long), 0, ctypes.byref(size)) == 0 and size.value > 0
    for ws, have in ((one, size.value - 1), (None, size.value), (264, size.value)):
        assert lib.rps_linear_attention_forward(ctypes.byref(long), *[one] * 8, ws, have, None) == -1
        assert b"workspace" in lib.rps_ops_last_error()
    nothing = ctypes.byref(attention_desc(sequences=0))
    assert lib.rps_linear_attention_forward(nothing, *[None] * 9, 0, None) == 0
    assert lib.rps_linear_attention_backward(nothing, *[None] * 13, 0, None) == 0
    for change in ({"sequences": 0}, {"tokens": 0}, {"sequences": 0, "tokens": 0}, {"sequences": 0, "tokens": 100_000}):
        for backward in (0, 1):
            assert lib.rps_linear_attention_workspace(ctypes.byref(attention_desc(**change)), backward, ctypes.byref(size)) == 0 and size.value == 0


def test_attention_refuses_cpu_tensors():
    from paper_1810_07766_b200 import ops

    q, ld = torch.zeros(2, 5, 3, 8), torch.zeros(3)
    with pytest.raises(ValueError, match="CUDA"):
        ops.linear_attention(q, q, q, ld)
    with pytest.raises(ValueError, match="CUDA"):
        ops.linear_attention_step(q[:, 0], q[:, 0], q[:, 0], ld, torch.zeros(2, 3, 8, 8))


def distil_desc(**changes):
    from paper_1810_07766_b200 import ops

    d = ops.rps_distil_desc(dtype=1, reduction=2, n=2, top_dtype=0, tokens=5, vocab=7, cols=8, top=3, ignore_index=-100, hidden_row=8, hidden_worker=40,
                            weight_row=8, weight_worker=56, dweight_row=8, dweight_worker=56, temperature=2.0)
    for k, v in changes.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change", [{"dtype": 2}, {"top_dtype": 2}, {"top_dtype": -1}, {"reduction": 3}, {"n": 0}, {"tokens": -1}, {"tokens": 1 << 24}, {"vocab": 0}, {"cols": 0},
                                    {"top": 0}, {"hidden_row": 7}, {"weight_row": 7}, {"hidden_worker": -1}, {"temperature": 0.0}, {"temperature": -1.0},
                                    {"temperature": float("nan")}, {"temperature": float("inf")}])
def test_distillation_descriptions_are_refused(lib, change):
    size, one = ctypes.c_size_t(), 256
    for backward in (0, 1):
        assert lib.rps_distil_workspace(ctypes.byref(distil_desc()), None, backward, ctypes.byref(size)) == 0 and size.value > 0
        assert lib.rps_distil_workspace(ctypes.byref(distil_desc(**change)), None, backward, ctypes.byref(size)) == -1
        assert lib.rps_ops_last_error()
    assert lib.rps_distil_forward(ctypes.byref(distil_desc(**change)), *[one] * 7, 1 << 30, None) == -1
    assert lib.rps_distil_backward(ctypes.byref(distil_desc(**change)), *[one] * 9, 1 << 30, None) == -1


def test_distillation_arrays_and_workspaces_are_refused(lib):
    from paper_1810_07766_b200 import ops

    size, one = ctypes.c_size_t(), 256
    assert lib.rps_distil_workspace(None, None, 0, ctypes.byref(size)) == -1
    assert lib.rps_distil_workspace(ctypes.byref(distil_desc()), None, 0, None) == -1
    assert lib.rps_distil_workspace(ctypes.byref(distil_desc(top=ops.MAX_TOP + 1)), None, 0, ctypes.byref(size)) == -5
    d = ctypes.byref(distil_desc())
    lib.rps_distil_workspace(d, one, 0, ctypes.byref(size))
    for at in range(7):
        args = [one] * 7
        args[at] = None
        assert lib.rps_distil_forward(d, *args, size.value, None) == -1, at
    assert lib.rps_distil_forward(d, *[one] * 7, size.value - 1, None) == -1 and b"workspace" in lib.rps_ops_last_error()
    lib.rps_distil_workspace(d, one, 1, ctypes.byref(size))
    for at in range(9):
        args = [one] * 9
        args[at] = None
        assert lib.rps_distil_backward(d, *args, size.value, None) == -1, at
    assert lib.rps_distil_backward(d, *[one] * 9, size.value - 1, None) == -1
    for change in ({"dweight_row": 7}, {"dweight_worker": 55}, {"dweight_worker": 0}):
        assert lib.rps_distil_backward(ctypes.byref(distil_desc(**change)), *[one] * 9, size.value, None) == -1
        assert b"dweight" in lib.rps_ops_last_error()


def test_distillation_refuses_cpu_tensors():
    from paper_1810_07766_b200 import ops

    h, w, ids = torch.zeros(4, 8), torch.zeros(6, 8), torch.zeros(4, 2, dtype=torch.int64)
    with pytest.raises(ValueError, match="CUDA"):
        ops.linear_distillation(h, w, ids, torch.zeros(4, 2))


def test_scales_beyond_fp32_are_refused(lib):
    size = ctypes.c_size_t()
    for scale, status in ((3.4e38, 0), (1e39, -1), (-1e300, -1)):
        assert lib.rps_embed_workspace(ctypes.byref(embed_desc(scale=scale)), ctypes.byref(size)) == status
        assert lib.rps_linear_attention_workspace(ctypes.byref(attention_desc(scale=scale)), 0, ctypes.byref(size)) == status
