"""Further host-side checks of the training operators, without a GPU."""
import ctypes

import pytest

from test_ops_host import lib  # noqa: F401


@pytest.mark.parametrize("change", [{"wait_limit_ms": -1}, {"withhold_sums": -1}, {"withhold_sums": 2}])
def test_norm_waits_are_described(lib, change):  # noqa: F811
    from paper_1810_07766_b200 import ops

    d = ops.rps_norm_desc(dtype=0, n=2, tokens=6, cols=10, gates=3, post_worker=10, pre_worker=10, gate_worker=30, scale=1.0, eps=1e-6, wait_limit_ms=5)
    size = ctypes.c_size_t()
    assert lib.rps_norm_workspace(ctypes.byref(d), ctypes.byref(size)) == 0
    for k, v in change.items():
        setattr(d, k, v)
    assert lib.rps_norm_workspace(ctypes.byref(d), ctypes.byref(size)) == -1 and b"wait_limit_ms" in lib.rps_ops_last_error()
