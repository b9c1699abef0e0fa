"""Refusals and no-ops of the calls around a block's Linears.  Arguments are checked on the host before anything is launched, so addresses that
nothing dereferences are enough and no GPU is needed."""
import ctypes as C
import math

import pytest

from paper_2603_25872_amd import drf

FAKE = 0x10000
EINVAL, ESHAPE, EUNSUPPORTED = -1, -2, -5
ref = lambda v: None if v is None else C.byref(v)  # noqa: E731


def rows(data=FAKE, slot=64 * 64, token=64):
    return drf.Rows(data, slot, token)


def norm(kind=drf.QK_LAYER, eps=1e-6, gain=None, bias=None):
    return drf.RowNorm(kind, eps, gain, bias)


def residual(x=rows(), y=rows(2 * FAKE), out=rows(), h=rows(2 * FAKE), **over):
    f = dict(stream=drf.F32, branch=drf.BF16, slots=2, tokens=64, width=64, lens=None, x_scale=1.0, y_scale=1.0, after=norm(drf.QK_NONE, 0.0), before=norm(),
             gate=rows(3 * FAKE, 64, 0), shift=rows(None), scale=rows(None))
    f.update(over)
    return drf.lib().drf_residual_norm(C.byref(drf.ResidualConfig(*(f[n] for n, _ in drf.ResidualConfig._fields_))), ref(x), ref(y), ref(out), ref(h), None)


def test_bad_residual_updates_are_refused():
    assert drf.lib().drf_residual_norm(None, *[C.byref(rows())] * 4, None) == EINVAL
    for over in (dict(stream=2), dict(branch=-1), dict(slots=-1), dict(tokens=-1), dict(width=0), dict(x_scale=math.inf), dict(y_scale=math.nan), dict(after=norm(3)),
                 dict(before=norm(-1)), dict(before=norm(eps=-1.0)), dict(after=norm(eps=math.nan)), dict(after=norm(drf.QK_NONE, 0.0, FAKE)),
                 dict(before=norm(drf.QK_RMS, 0.0, FAKE, FAKE))):
        assert residual(**over) == EINVAL
        assert len(drf.lib().drf_last_error()) > 0
    assert residual(stream=drf.BF16, branch=drf.F32) == EUNSUPPORTED
    assert residual(width=16385) == residual(tokens=2 ** 30 + 1) == residual(slots=2 ** 15, tokens=2 ** 15 + 1) == residual(slots=2 ** 31 - 1, tokens=2 ** 30) == ESHAPE
    for bad in (dict(x=None), dict(x=rows(None)), dict(y=rows(None)), dict(out=rows(None)), dict(h=rows(None)), dict(out=None, h=None), dict(y=None)):
        assert residual(**bad) == EINVAL
    for bad in (dict(out=rows(token=128)), dict(h=rows(2 * FAKE, slot=64)), dict(out=rows(2 * FAKE)), dict(h=rows()), dict(out=rows(5 * FAKE), h=rows(5 * FAKE))):
        assert residual(**bad) == EINVAL                                        # an output on another tensor, or on its own in another layout
    assert residual(tokens=0, x=None, y=None, out=None, h=None) == residual(slots=0, x=None, y=None, out=None, h=None) == 0


@pytest.mark.parametrize("bad", [dict(slot=0), dict(token=0), dict(token=32), dict(token=-63), dict(slot=8)])
def test_outputs_whose_rows_lie_on_one_another_are_refused(bad):
    assert residual(out=rows(7 * FAKE, **bad)) == residual(h=rows(7 * FAKE, **bad)) == EINVAL
    assert ffn(out=rows(7 * FAKE, **bad)) == adapters(out=rows(7 * FAKE, **bad)) == (ESHAPE if bad.get("token", 0) < 0 else EINVAL)


def ffn_config(**over):
    f = dict(dtype=drf.BF16, act=0, slots=2, tokens=64, width=64, hidden=128, out_width=64, lens=None, w_in=FAKE, w_out=FAKE, b_in=None, b_out=None)
    f.update(over)
    return drf.GatedFfnConfig(*(f[n] for n, _ in drf.GatedFfnConfig._fields_))


def ffn(x=rows(), out=rows(2 * FAKE), scratch=FAKE, n=1 << 40, **over):
    return drf.lib().drf_gated_ffn(C.byref(ffn_config(**over)), ref(x), ref(out), scratch, n, None)


def adapters_config(**over):
    f = dict(dtype=drf.BF16, slots=2, tokens=64, width=64, out_width=64, rank=8, adapters=3, lens=None, which=FAKE, w=FAKE, a=FAKE, b=FAKE, bias=None, scales=None)
    f.update(over)
    return drf.AdaptersConfig(*(f[n] for n, _ in drf.AdaptersConfig._fields_))


def adapters(x=rows(), out=rows(2 * FAKE), scratch=FAKE, n=1 << 40, **over):
    return drf.lib().drf_linear_adapters(C.byref(adapters_config(**over)), ref(x), ref(out), scratch, n, None)


@pytest.mark.parametrize("call", [ffn, adapters])
def test_bad_linears_are_refused(call):
    for over in (dict(dtype=2), dict(slots=-1), dict(tokens=-1), dict(width=0), dict(out_width=0), dict(x=None), dict(out=None), dict(x=rows(None)), dict(out=rows(None)),
                 dict(scratch=None), dict(scratch=FAKE + 8), dict(n=1), dict(out=rows())):
        assert call(**over) == EINVAL
        assert len(drf.lib().drf_last_error()) > 0
    for over in (dict(tokens=2 ** 30 + 1), dict(slots=2 ** 16, tokens=2 ** 15), dict(width=2 ** 20 + 8), dict(out_width=2 ** 20 + 1), dict(width=60), dict(x=rows(FAKE + 2)),
                 dict(x=rows(token=68)), dict(x=rows(slot=68)), dict(x=rows(token=1 << 22)), dict(x=rows(token=-64)), dict(out=rows(2 * FAKE, slot=-4096)),
                 dict(out=rows(2 * FAKE, token=1 << 22))):
        assert call(**over) == ESHAPE
    for none in (dict(slots=0), dict(tokens=0)):
        assert call(x=None, out=None, scratch=None, n=0, **none) == 0


def test_bad_feed_forwards_are_refused():
    assert drf.lib().drf_gated_ffn(None, *[C.byref(rows())] * 2, FAKE, 1 << 40, None) == EINVAL
    assert ffn(act=2) == ffn(hidden=0) == ffn(w_in=None) == ffn(w_out=None) == EINVAL
    assert ffn(hidden=132) == ffn(hidden=2 ** 20 + 8) == ffn(w_in=FAKE + 8) == ffn(w_out=FAKE + 8) == ESHAPE


def test_bad_adapters_are_refused():
    assert drf.lib().drf_linear_adapters(None, *[C.byref(rows())] * 2, FAKE, 1 << 40, None) == EINVAL
    assert adapters(rank=0) == adapters(adapters=-1) == adapters(w=None) == adapters(a=None) == adapters(b=None) == adapters(which=None) == EINVAL
    assert adapters(rank=257) == adapters(w=FAKE + 8) == adapters(a=FAKE + 8) == ESHAPE


def test_scratch():
    f = lambda **over: drf.lib().drf_gated_ffn_scratch_bytes(C.byref(ffn_config(**over)))  # noqa: E731
    assert f() >= 2 * 64 * 128 * 2 and f(dtype=drf.F32) >= 2 * 64 * 128 * 4
    assert f(dtype=5) == f(slots=0) == f(hidden=4) == f(width=0) == f(tokens=-1) == drf.lib().drf_gated_ffn_scratch_bytes(None) == 0
    g = lambda **over: drf.lib().drf_linear_adapters_scratch_bytes(C.byref(adapters_config(**over)))  # noqa: E731
    assert g() >= 2 * 64 * 8 * 4
    assert g(adapters=0) == g(rank=300) == g(slots=0) == g(width=-8) == drf.lib().drf_linear_adapters_scratch_bytes(None) == 0
    assert ffn(n=f() - 1) == adapters(n=g() - 1) == EINVAL


def test_binding_refuses_what_it_cannot_describe():
    import torch
    x, w, i = torch.zeros(1, 4, 8), torch.zeros(16, 8), torch.zeros(1, dtype=torch.int32)
    for call in (lambda: drf.residual_norm(x, x), lambda: drf.gated_ffn(x, w, w.t().contiguous()), lambda: drf.linear_adapters(x, w, w[None, :2], w[None, :, :2], i)):
        with pytest.raises(AssertionError):                                     # host tensors: there is no CPU fallback
            call()
