"""Scales that the cache's calls refuse: those that are not finite in log2 units."""
import pytest

from test_cache_host import B, _attend, _dims, _views  # noqa: F401 (B: a fixture)


@pytest.mark.parametrize("scale", [2.5e38, 3.0e38, 3.4e38, float("inf"), float("nan"), -1e-45])
def test_scales_beyond_log2_units_are_refused(B, scale):
    import ctypes
    d = _dims(B)
    q, pre, own = _views(B, d)
    assert _attend(B, d, q, pre, pre, own, own, scale=scale) == B.ERR_INVALID_ARG
    assert B.lib().brisk_cache_weights(ctypes.byref(d), ctypes.byref(q), 256, ctypes.byref(own), 256, None, scale, 1.0,
                                       None, 256, 256, None) == B.ERR_INVALID_ARG
