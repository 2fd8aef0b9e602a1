"""Exact attention's host side (no GPU): refusals of values that the kernels' arithmetic has no room for."""
import math

import pytest

import paper_2201_12854_amd as mca
from paper_2201_12854_amd import binding
from test_exact_host import _backward, _desc, _forward, _size


@pytest.mark.parametrize("dtype", [binding.MCA_F32, binding.MCA_BF16])
@pytest.mark.parametrize("scale", [math.nextafter(2.0 ** -100, 0), 1e-35, 1e-38, 1e-40])
def test_small_scales_refused(dtype, scale):
    for backward in (0, 1):
        assert _size(_desc(dtype=dtype, scale=2.0 ** -100), backward)[0] == binding.MCA_OK
        assert _size(_desc(dtype=dtype, scale=scale), backward)[0] == binding.MCA_ERR_INVALID_ARGUMENT
    assert _forward(_desc(dtype=dtype, scale=scale)) == binding.MCA_ERR_INVALID_ARGUMENT
    assert _backward(_desc(dtype=dtype, scale=scale)) == binding.MCA_ERR_INVALID_ARGUMENT
    assert "2^-100" in mca.load_library().mca_last_error().decode()


def test_wide_window_refused():
    """Not taken modulo 2^64, where 2^64 + 2 would be a window of 2 and 2^64 none."""
    for window in (2**64, 2**64 + 2, 2**63, -2**63 - 2):
        with pytest.raises(ValueError):
            binding._int64("window", window)
    assert binding._int64("window", 256) == 256 and binding._int64("window", -2**63) == -2**63
