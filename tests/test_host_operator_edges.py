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


@pytest.mark.parametrize("over", [dict(slot=0), dict(token=0), dict(head=0), dict(head=32), dict(token=-56), dict(slot=8)])
@pytest.mark.parametrize("dtype", [drf.BF16, drf.F32])
def test_outputs_whose_rows_lie_on_one_another_are_refused(over, dtype):
    """(Every row would be written by several workgroups at once.)  As inputs they are calls like others; of a dimension of one element no stride counts."""
    L, x, y, rc, s = drf.lib(), heads(), heads(2 * FAKE, **over), config(), shape(dtype=dtype)
    ref = C.byref
    assert L.drf_rope(ref(rc), dtype, 2, 64, 4, 64, None, None, 0, ref(x), ref(y), None) == EINVAL
    cfg = drf.QkConfig(drf.QK_RMS, 1e-6, 1.0)
    for outs in ((y, x), (x, y)):
        assert L.drf_qk_norm_rope(ref(cfg), ref(rc), ref(s), None, 0, ref(x), ref(x), ref(outs[0]), ref(outs[1]), None) == EINVAL
    assert attend(s, out=y) == (ESHAPE if over.get("token", 0) < 0 else EINVAL)
    assert L.drf_rope(ref(rc), dtype, 0, 64, 4, 64, None, None, 0, ref(x), ref(y), None) == 0


def test_more_tiles_than_a_launch_has_are_refused():
    """On the host, before a device is asked for anything."""
    L, t = drf.lib(), heads(slot=64 * 4 * 128, token=4 * 128, head=128)
    for q_block in (32, 64, 128):
        for dtype, tokens in ((drf.BF16, 1 << 26), (drf.F32, 1 << 23)):
            for head_dim in (8, 64, 72, 128):
                s = shape(dtype=dtype, slots=1 << 7, q_tokens=tokens, head_dim=head_dim)
                assert L.drf_block_attention(C.byref(s), q_block, 64, C.c_float(1.0), FAKE, *[C.byref(t)] * 4, None) == ESHAPE
    for s in (shape(slots=1 << 23), shape(slots=1 << 19, q_heads=16, kv_heads=16), shape(q_tokens=1 << 30)):
        assert L.drf_block_select(C.byref(s), 32, 64, 4, C.byref(t), C.byref(t), FAKE, 1 << 62, FAKE, None) == ESHAPE
