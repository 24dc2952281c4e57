"""The workspace of shared-prefix attention: one that is large enough for a batch is for
every smaller one, whatever the division of the work."""
import ctypes

import pytest

from paper_2504_15299_amd import api


def need(*a):
    n = ctypes.c_size_t()
    assert api.lib().d2moe_attn_prefix_workspace(*a, ctypes.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("heads", [(32, 8, 128), (12, 12, 64), (34, 2, 256), (1, 1, 8),
                                   (64, 1, 128)])
@pytest.mark.parametrize("lengths", [(8192, 512), (8192, 0), (0, 5000), (129, 65),
                                     (1 << 30, 1 << 30)])
def test_grows_with_the_batch(heads, lengths):
    last = 0
    for B in list(range(1, 700)) + list(range(700, 65000, 331)):
        now = need(B, *heads, *lengths)
        assert now >= last, (B, last, now)
        last = now

