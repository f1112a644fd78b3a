"""Bases so small that a frequency is no number."""
import ctypes

import pytest

from test_prompt_host import H  # noqa: F401 (fixture)


@pytest.mark.parametrize("base", [5e-324, 1e-318])
@pytest.mark.parametrize("scaling", [0, 1, 3])
def test_frequencies_past_the_largest_number_are_refused(H, base, scaling):
    p = H.hkv_rope_params(128, 128, 0, 1, (ctypes.c_int32 * 3)(64), 0, scaling, 0, base, 2.0, 100.0, 1.0, 32.0, 1.0)
    rope = H.hkv_rope()
    rope.rot_dim = 7
    assert H.lib().hkv_make_rope(ctypes.addressof(p), ctypes.addressof(rope)) == H.HKV_ERR_INVALID_ARG
    assert rope.rot_dim == 7    # left as it was
    # half of the way there it is one
    p.base = 1e-300
    assert H.lib().hkv_make_rope(ctypes.addressof(p), ctypes.addressof(rope)) == H.HKV_OK and rope.rot_dim == 128
