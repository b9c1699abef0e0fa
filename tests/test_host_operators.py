"""Refusals and no-ops of the attention operators' calls.  Arguments are checked on the host before anything is launched, so addresses that
nothing dereferences are enough and no GPU is needed."""
import ctypes as C
import math

import pytest

from paper_2603_25872_amd import drf

FAKE = 0x10000
EINVAL, ESHAPE = -1, -2


def heads(data=FAKE, slot=64 * 4 * 64, token=4 * 64, head=64):
    return drf.Heads(data, slot, token, head)


def shape(**over):
    f = dict(dtype=drf.BF16, slots=2, q_tokens=64, kv_tokens=64, q_heads=4, kv_heads=4, head_dim=64, q_lens=None, kv_lens=None)
    f.update(over)
    return drf.AttnShape(*(f[n] for n, _ in drf.AttnShape._fields_))


def config(**over):
    rc = drf.rope_config((32, 32), (8, 8))
    for k, v in over.items():
        if isinstance(v, tuple):
            getattr(rc, k)[v[0]] = v[1]
        else:
            setattr(rc, k, v)
    return rc


def rope(rc, dtype=drf.BF16, slots=2, tokens=64, n_heads=4, d=64, x=None, out=None):
    ref = lambda s: None if s is None else C.byref(s)  # noqa: E731
    return drf.lib().drf_rope(ref(rc), dtype, slots, tokens, n_heads, d, None, None, 0, ref(x), ref(out), None)


def qk(cfg, rc, s, q=heads(), k=heads(), qo=heads(), ko=heads()):
    ref = lambda v: None if v is None else C.byref(v)  # noqa: E731
    return drf.lib().drf_qk_norm_rope(ref(cfg), ref(rc), ref(s), None, 0, ref(q), ref(k), ref(qo), ref(ko), None)


@pytest.mark.parametrize("over,status", [
    (dict(n_axes=0), EINVAL), (dict(n_axes=4), EINVAL), (dict(theta=0.0), EINVAL), (dict(theta=-1.0), EINVAL), (dict(theta=math.inf), EINVAL),
    (dict(theta=math.nan), EINVAL), (dict(layout=2), EINVAL), (dict(dim=(0, 31)), EINVAL), (dict(dim=(1, -2)), EINVAL), (dict(dim=(1, 34)), ESHAPE),
    (dict(dim=(0, 2 ** 31 - 2)), ESHAPE), (dict(extent=(1, 0)), EINVAL), (dict(origin=(0, math.nan)), EINVAL), (dict(step=(1, math.inf)), EINVAL)])
def test_bad_rotations_are_refused(over, status):
    x = heads()
    assert rope(config(**over), x=x, out=x) == status
    assert len(drf.lib().drf_last_error()) > 0
    assert qk(drf.QkConfig(drf.QK_RMS, 1e-6, 1.0), config(**over), shape()) == status


def test_bad_rope_arguments_are_refused():
    x, rc = heads(), config()
    assert rope(None, x=x, out=x) == EINVAL
    for over in (dict(dtype=7), dict(slots=-1), dict(tokens=-1), dict(n_heads=0), dict(d=0)):
        assert rope(rc, x=x, out=x, **over) == EINVAL
    assert rope(rc, x=x, out=x, d=136) == ESHAPE
    for bad in (dict(x=None, out=x), dict(x=x, out=None), dict(x=heads(data=None), out=x), dict(x=x, out=heads(data=None))):
        assert rope(rc, **bad) == EINVAL
    assert rope(rc, x=x, out=heads(token=8 * 64)) == EINVAL                     # one address, two layouts
    for none in (dict(slots=0), dict(tokens=0)):
        assert rope(rc, x=None, out=None, **none) == 0


def test_bad_norms_are_refused():
    ok, rc = drf.QkConfig(drf.QK_RMS, 1e-6, 1.0), config()
    assert qk(None, rc, shape()) == qk(ok, rc, None) == EINVAL
    for cfg in (drf.QkConfig(3, 1e-6, 1.0), drf.QkConfig(drf.QK_RMS, -1e-6, 1.0), drf.QkConfig(drf.QK_RMS, math.nan, 1.0),
                drf.QkConfig(drf.QK_RMS, 1e-6, math.inf), drf.QkConfig(drf.QK_NONE, 0.0, 1.0, FAKE), drf.QkConfig(drf.QK_NONE, 0.0, 1.0, None, None, FAKE),
                drf.QkConfig(drf.QK_RMS, 0.0, 1.0, FAKE, FAKE), drf.QkConfig(drf.QK_RMS, 0.0, 1.0, None, None, None, FAKE)):
        assert qk(cfg, rc, shape()) == EINVAL
    for over in (dict(kv_tokens=63), dict(kv_lens=FAKE), dict(q_lens=FAKE, kv_lens=FAKE + 64), dict(dtype=2), dict(kv_heads=0)):
        assert qk(ok, rc, shape(**over)) == EINVAL
    for bad in (dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(k=heads(data=None)), dict(ko=heads(head=128))):
        assert qk(ok, rc, shape(), **bad) == EINVAL
    assert qk(ok, rc, shape(slots=0), None, None, None, None) == qk(ok, None, shape(q_tokens=0, kv_tokens=0), None, None, None, None) == 0


def test_block_words_and_scratch():
    L = drf.lib()
    assert [L.drf_block_words(n, 32) for n in (0, 1, 32, 1024, 1025)] == [0, 1, 1, 1, 2]
    assert L.drf_block_words(4096, 128) == 1 and L.drf_block_words(2 ** 31 - 1, 128) == 2 ** 19
    assert L.drf_block_words(-1, 64) == L.drf_block_words(64, 48) == 0
    need = lambda s, qb=64, kb=64: L.drf_block_select_scratch_bytes(C.byref(s), qb, kb)  # noqa: E731
    assert need(shape()) == 2 * (4 + 4) * 16 * 64 * 8                             # one tile of 16 blocks a head
    assert need(shape(q_tokens=2000, head_dim=61)) == 2 * 4 * (32 + 16) * 64 * 8   # columns padded to eight
    assert need(shape(), 16) == need(shape(dtype=5)) == need(shape(head_dim=129)) == L.drf_block_select_scratch_bytes(None, 64, 64) == 0


def test_bad_selections_are_refused():
    L, t = drf.lib(), heads()
    call = lambda s, qb=64, kb=64, topk=4, q=t, k=t, scratch=FAKE, n=1 << 20, out=FAKE: L.drf_block_select(  # noqa: E731
        None if s is None else C.byref(s), qb, kb, topk, None if q is None else C.byref(q), None if k is None else C.byref(k), scratch, n, out, None)
    assert call(None) == EINVAL
    for over in (dict(qb=0), dict(qb=96), dict(kb=256), dict(topk=0), dict(topk=-1), dict(q=None), dict(k=heads(data=None)), dict(scratch=None),
                 dict(out=None), dict(scratch=FAKE + 8), dict(n=2 * (4 + 4) * 16 * 64 * 8 - 1)):
        assert call(shape(), **over) == EINVAL
    assert call(shape(q_heads=6)) == call(shape(head_dim=136)) == ESHAPE
    assert call(shape(kv_tokens=1025 * 32), kb=32) == ESHAPE                       # more key blocks than are compared
    assert call(shape(dtype=9)) == call(shape(slots=-1)) == EINVAL
    for none in (dict(slots=0), dict(q_tokens=0), dict(kv_tokens=0)):
        assert call(shape(**none), q=None, k=None, scratch=None, n=0, out=None) == 0


def test_bad_attentions_are_refused():
    L, t = drf.lib(), heads()
    ref = lambda v: None if v is None else C.byref(v)  # noqa: E731
    call = lambda s, qb=64, kb=64, scale=0.125, blocks=FAKE, q=t, k=t, v=t, out=t: L.drf_block_attention(  # noqa: E731
        ref(s), qb, kb, C.c_float(scale), blocks, ref(q), ref(k), ref(v), ref(out), None)
    assert call(None) == EINVAL
    for over in (dict(qb=1), dict(kb=63), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(blocks=None), dict(q=None),
                 dict(k=None), dict(v=heads(data=None)), dict(out=None)):
        assert call(shape(), **over) == EINVAL
    for bad in (heads(data=FAKE + 8), heads(head=60), heads(token=4 * 64 + 4), heads(slot=4), heads(token=1 << 24), heads(token=-256)):
        for name in ("q", "k", "v", "out"):
            assert call(shape(), **{name: bad}) == ESHAPE
    assert call(shape(head_dim=60)) == call(shape(head_dim=136)) == call(shape(kv_heads=3)) == ESHAPE
    assert call(shape(q_heads=0)) == EINVAL
    assert call(shape(slots=0), q=None, k=None, v=None, out=None, blocks=None) == call(shape(q_tokens=0), q=None, out=None) == 0


def test_scratch_of_split_attentions():
    L, t = drf.lib(), heads()
    need = lambda s: L.drf_block_attention_scratch_bytes(None if s is None else C.byref(s))  # noqa: E731
    long = dict(slots=1, q_tokens=1, kv_tokens=8192)
    assert need(shape(**long)) == 4 * 8 * 32 * 68 * 4                              # a tile a head, eight workgroups each
    assert need(shape(**dict(long, kv_tokens=1 << 20))) == 4 * 64 * 32 * 68 * 4    # a workgroup a CU
    assert need(shape(**dict(long, kv_tokens=8191))) == need(shape(**dict(long, q_tokens=513))) == need(shape(**dict(long, dtype=0))) == 0
    assert need(None) == need(shape(**dict(long, slots=0))) == need(shape(**dict(long, q_tokens=0))) == need(shape(**dict(long, head_dim=136))) == 0
    call = lambda scratch, n: L.drf_block_attention_split(C.byref(shape(**long)), 64, 64, C.c_float(1.0), FAKE, *[C.byref(t)] * 4, scratch, n, None)  # noqa: E731
    assert call(FAKE + 4, 1 << 30) == call(FAKE, 4 * 8 * 32 * 68 * 4 - 1) == call(FAKE, 0) == EINVAL


@pytest.mark.parametrize("tokens", [2 ** 30 + 1, 2 ** 31 - 1])
def test_more_tokens_than_are_counted_are_refused(tokens):
    """Sizes whose tiles, rounded up, would not fit 32 bits."""
    L, t = drf.lib(), heads()
    rc, cfg = drf.rope_config((64,), (1,)), drf.QkConfig(norm=0, q_scale=1.0)
    assert L.drf_rope(C.byref(rc), 1, 1, tokens, 4, 64, None, None, 0, C.byref(t), C.byref(t), None) == ESHAPE
    s = shape(q_tokens=tokens, kv_tokens=tokens)
    assert L.drf_qk_norm_rope(C.byref(cfg), C.byref(rc), C.byref(s), None, 0, *[C.byref(t)] * 4, None) == ESHAPE
    for over in (dict(q_tokens=tokens), dict(kv_tokens=tokens)):
        assert L.drf_block_attention(C.byref(shape(**over)), 64, 64, C.c_float(1.0), FAKE, *[C.byref(t)] * 4, None) == ESHAPE
    assert L.drf_block_select(C.byref(shape(q_tokens=tokens)), 32, 64, 4, C.byref(t), C.byref(t), FAKE, 1 << 62, FAKE, None) == ESHAPE


def test_binding_refuses_what_it_cannot_describe():
    import torch
    x = torch.zeros(1, 4, 2, 8)
    rc = drf.rope_config((4, 4), (2, 2))
    for call in (lambda: drf.rope(x, rc), lambda: drf.qk_norm_rope(x, x, "rms", rc), lambda: drf.block_select(x, x, 32, 32, 1),
                 lambda: drf.block_attention(x, x, x, torch.zeros(1, 2, 1, 1, dtype=torch.int32), 32, 32)):
        with pytest.raises(AssertionError):                                     # host tensors: there is no CPU fallback
            call()
    for dims, extents in (((), ()), ((2, 2, 2, 2), (1, 1, 1, 1)), ((4, 4), (2,))):
        with pytest.raises(ValueError):
            drf.rope_config(dims, extents)
    with pytest.raises(KeyError):
        drf.rope_config((4,), (2,), layout="spiral")
