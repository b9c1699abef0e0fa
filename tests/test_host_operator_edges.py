"""More refusals of the attention operators' calls, on the host: arguments are checked before anything is launched."""
import ctypes as C

import pytest

from paper_2603_25872_amd import drf
from test_host_operators import EINVAL, ESHAPE, FAKE, config, heads, shape


def attend(s, scale=0.125, **over):
    t = dict(dict(q=heads(), k=heads(), v=heads(), out=heads()), **over)
    return drf.lib().drf_block_attention(C.byref(s), 64, 64, C.c_float(scale), FAKE, *[C.byref(t[n]) for n in ("q", "k", "v", "out")], None)


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_a_scale_that_is_no_number_in_exponents_of_two_is_refused(scale):
    assert attend(shape(), scale) == EINVAL


def test_more_workgroups_than_are_numbered_are_refused():
    x, rc = heads(), config()
    assert drf.lib().drf_rope(C.byref(rc), drf.BF16, 1 << 20, 1 << 30, 4, 64, None, None, 0, C.byref(x), C.byref(x), None) == ESHAPE
