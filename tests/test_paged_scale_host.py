"""The attention's scale at the end of fp32's range (no GPU needed: refused before any device work)."""
import ctypes

import pytest

import paper_2503_05130_amd as ie

P = 1 << 20          # stands for an aligned device address; nothing here reads it


@pytest.mark.parametrize("scale", [3e38, -3e38, 2.4e38, float("inf"), float("-inf"), float("nan")])
def test_scales_that_overflow_in_powers_of_two_are_refused(scale):
    c = ie.PagedCacheDesc(ie.ABI_VERSION, ie.KV_BF16, 10, 16, 4, 64, P, 2 * P, None, None)
    assert ie.lib().iefwd_paged_attention(ctypes.byref(c), P, 512, 8, P, 10, 10, P, 3, scale, P, P, 1 << 20, None) == ie.EINVAL
    assert "scale" in ie.last_error()
