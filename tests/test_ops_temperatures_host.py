"""Which temperatures distillation takes; needs no GPU."""
import ctypes

import pytest

from test_ops_sequence_host import distil_desc, lib  # noqa: F401


@pytest.mark.parametrize("temperature,status", [(0.01, 0), (1.0, 0), (100.0, 0), (0.009999999776482582, 0), (0.0099, -1), (1e-6, -1), (100.1, -1), (1e6, -1)])
def test_temperatures_whose_losses_fp32_holds(lib, temperature, status):  # noqa: F811
    size = ctypes.c_size_t()
    for backward in (0, 1):
        assert lib.rps_distil_workspace(ctypes.byref(distil_desc(temperature=temperature)), None, backward, ctypes.byref(size)) == status
        assert (b"temperature" in lib.rps_ops_last_error()) == (status != 0)
