"""Heads without columns are refused like any other wrong shape; needs no GPU."""
import ctypes

import pytest
import torch

from test_ops_sequence_host import attention_desc, lib  # noqa: F401


@pytest.mark.parametrize("shape", [(2, 5, 3, 0), ()])
def test_queries_without_columns_are_no_division_by_zero(lib, shape):  # noqa: F811
    from paper_1810_07766_b200 import ops

    q, v, ld = torch.zeros(shape), torch.zeros(2, 5, 3, 8), torch.zeros(3)
    with pytest.raises(ValueError, match="CUDA"):
        ops.linear_attention(q, q, v, ld)
    size = ctypes.c_size_t()
    assert lib.rps_linear_attention_workspace(ctypes.byref(attention_desc(key_cols=0)), 0, ctypes.byref(size)) == -1 and b"key_cols" in lib.rps_ops_last_error()
