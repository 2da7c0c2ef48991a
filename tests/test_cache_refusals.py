"""What attention over the 4-bit cache refuses beyond the shapes of tests/test_cache_abi.py, without a GPU."""
import ctypes

import pytest

from test_cache_abi import A, B_, BIG, EINVAL, P, _cache, _shape  # noqa: F401  (P is the fixture)


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38, float("inf")])
def test_a_scale_that_is_no_number_in_units_of_log2(P, scale):
    """the logits are multiplied with scale * log2(e), which is beyond binary32 here"""
    L = P.load_library()
    c, s = ctypes.byref(_cache(P).c()), ctypes.byref(_shape(P, scale=scale).c())
    assert L.pasa_cache_attn_workspace_bytes(s, c, 0) == 0
    assert L.pasa_cache_attn(A, s, c, A, BIG, A, A, None, 0, 0, B_, None, A, BIG, None) == EINVAL


def test_the_largest_scale(P):
    c, s = ctypes.byref(_cache(P).c()), ctypes.byref(_shape(P, scale=2.3e38).c())
    assert P.load_library().pasa_cache_attn_workspace_bytes(s, c, 0) > 0
