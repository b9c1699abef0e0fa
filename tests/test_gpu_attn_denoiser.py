"""Denoisers with norms, rotations and chosen key blocks in their self-attention: against the definitions in float64, and through every call
that takes a handle."""
import numpy as np
import pytest

from paper_2603_25872_amd import drf as D_, inputs as I
from attn_reference import dit as reference
from parity import TOL_BF16, TOL_F32, check

ROPE = dict(rope_dim=(16, 16))
CASES = {
    # name: (model over configuration 1's, attention operators, slots)
    "f32-rms-rope": (dict(), dict(qk_norm="rms", **ROPE), 3),
    "f32-layer-halves": (dict(), dict(qk_norm="layer", rope_dim=(8, 24), rope_layout="halves", additive_pos=False, norm_eps=1e-3), 2),
    "f32-rope-only": (dict(lat_h=10, lat_w=14), dict(rope_dim=(12, 6), rope_theta=100.0), 2),
    "f32-blocks": (dict(lat_h=24, lat_w=26), dict(blocks=(128, 64, 2)), 1),
    "f32-all": (dict(lat_h=24, lat_w=26), dict(qk_norm="rms", blocks=(64, 64, 2), **ROPE), 1),
    "bf16-rms-rope": (dict(dtype=I.BF16, hidden=192, heads=3), dict(qk_norm="rms", rope_dim=(32, 32)), 3),
    # head width 72, and enough workgroups that the attention wants its queries scaled
    "bf16-xl-width": (dict(dtype=I.BF16, hidden=576, heads=8, lat_h=36, lat_w=36), dict(qk_norm="rms", rope_dim=(36, 36)), 8),
    "bf16-layer-all-blocks": (dict(dtype=I.BF16, hidden=192, heads=3, lat_h=24, lat_w=26), dict(qk_norm="layer", rope_dim=(32, 32), blocks=(64, 32, 5)), 2),
    "bf16-text-blocks": (dict(dtype=I.BF16, hidden=192, heads=3, lat_h=24, lat_w=26, cond=I.COND_TEXT, cond_dim=64, ctx_len=9),
                         dict(qk_norm="rms", rope_dim=(32, 32), blocks=(128, 64, 2)), 1),
    # a width that blocks of one launch take without these operators
    "bf16-narrow": (dict(dtype=I.BF16, hidden=256, heads=4), dict(qk_norm="rms", additive_pos=False, rope_dim=(32, 32)), 3),
    "bf16-no-code": (dict(dtype=I.BF16, hidden=256, heads=4), dict(additive_pos=False), 3),
}


def model(name):
    over, attn, slots = CASES[name]
    return dict(I.config(1)["dit"], attn=attn, **over), slots


def inputs_of(dit, slots, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((slots, dit["in_ch"], dit["lat_h"], dit["lat_w"])).astype(np.float32)
    t = rng.integers(0, 1000, slots).astype(np.int32)
    shape = (slots, dit["ctx_len"], dit["cond_dim"]) if dit["cond"] == I.COND_TEXT else (slots, dit["cond_dim"])
    return x, t, rng.standard_normal(shape).astype(np.float32)


def rounded(w):
    """To bf16, as a bf16 handle takes its parameters."""
    u = w.view(np.uint32).astype(np.uint64)
    return ((u + 0x7fff + ((u >> 16) & 1)) & 0xffff0000).astype(np.uint32).view(np.float32)


def expected(name):
    dit, slots = model(name)
    w = I.weights(dit, 7, "loud")
    x, t, c = inputs_of(dit, slots, 8)
    margins = []
    wr, cr = (rounded(w), rounded(c) if dit["cond"] == I.COND_TEXT else c) if dit["dtype"] == I.BF16 else (w, c)
    return dit, w, x, t, c, reference(dit, wr, x, t, cr, margins), margins


@pytest.mark.parametrize("name", [n for n, c in CASES.items() if "blocks" in c[1]])
def test_choices_of_the_cases_are_clear(name):
    """The blocks that a case chooses do not hang on a rounding: q and k are off by 2^-8 in bf16 and 2^-20 in fp32, means of 32 and more rows of
    them by a fraction of that; a margin of 2^-6 (2^-12) of the scores' spread is several times it."""
    dit, _, _, _, _, _, margins = expected(name)
    assert all(m > (2.0 ** -6 if dit["dtype"] == I.BF16 else 2.0 ** -12) for m in margins), margins


def test_weight_counts_and_refusals():
    base = I.config(1)["dit"]
    assert D_.denoiser_weight_count(dict(base, attn=dict())) == D_.denoiser_weight_count(base) == I.param_count(base)
    for name in CASES:
        dit, _ = model(name)
        assert D_.denoiser_weight_count(dit) == I.param_count(dit) > 0
    for bad in (dict(rope_dim=(16, 18)), dict(rope_dim=(3, 4)), dict(rope_dim=(-2, 4)), dict(rope_dim=(4, 4), rope_theta=0.0), dict(qk_norm="rms", norm_eps=-1.0),
                dict(additive_pos=2), dict(blocks=(64, 64, -1)), dict(blocks=(0, 0, 1)), dict(blocks=(64, 48, 1))):
        assert D_.denoiser_weight_count(dict(base, attn=bad)) == 0
    assert D_.denoiser_weight_count(dict(base, lat_h=1024, lat_w=1024, attn=dict(blocks=(128, 128, 8)))) == 0       # 2048 key blocks


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available()
    return t


@pytest.mark.gpu
@pytest.mark.parametrize("name", CASES)
def test_denoiser_against_the_definition(torch, name):
    dit, w, x, t, c, want, _ = expected(name)
    den = D_.Denoiser(dit, w)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    got = den.eps_batched(dev(x), dev(t), dev(c))
    check(got.cpu().numpy(), want, TOL_BF16 if dit["dtype"] == I.BF16 else TOL_F32, name)
    few = [dev(a[:3]) for a in (x, t, c)]                                       # what fits the static scratch array
    static = torch.full_like(few[0], float("nan"))
    den.eps_batched_static(*few, static)
    assert torch.equal(static, den.eps_batched(*few))
    den.profile_enable(1)
    assert torch.equal(den.eps_batched(dev(x), dev(t), dev(c)), got)
    # (a block of one launch counts as GEMM with the attention in it)
    assert den.profile_read(D_.PROF_ATTN if name != "bf16-no-code" else D_.PROF_GEMM)["work"] > 0
    den.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [I.F32, I.BF16])
def test_nothing_in_it_is_the_plain_denoiser(torch, dtype):
    dit = dict(I.config(1)["dit"], dtype=dtype)
    w = I.weights(dit, 7, "loud")
    x, t, c = (torch.from_numpy(a).cuda() for a in inputs_of(dit, 3, 9))
    a, b = D_.Denoiser(dit, w), D_.Denoiser(dict(dit, attn=dict()), w)
    one = a.eps_batched(x, t, c)
    torch.cuda.synchronize()
    assert torch.equal(b.eps_batched(x, t, c), one)
    torch.cuda.synchronize()
    a.close()
    b.close()


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["f32-all", "bf16-text-blocks", "bf16-xl-width"])
def test_sampling_eager_and_replayed(torch, name):
    """Draft-and-refine sampling: kernel by kernel, captured and replayed give the same bits; n = 1 is sequential in both modes."""
    dit, _ = model(name)
    den = D_.Denoiser(dit, I.weights(dit, 7, "loud"))
    sched = dict(I.config(1)["sched"], steps=6)
    xT, _, c = (torch.from_numpy(a).cuda() for a in inputs_of(dit, 2, 10))
    outs = {}
    for mode in (I.CONSERVATIVE, I.AGGRESSIVE):
        for n in (1, 3):
            den.use_graphs(0)
            want = den.sample(sched, mode, n, xT, c)
            den.use_graphs(2)
            out = torch.empty_like(xT)
            for _ in range(3):
                out.fill_(float("nan"))
                den.sample(sched, mode, n, xT, c, out=out)
                torch.cuda.synchronize()
                assert torch.equal(out, want) and torch.isfinite(out).all()
                den.eps_batched(xT, torch.zeros(2, dtype=torch.int32, device="cuda"), c)
            outs[mode, n] = want
    assert den.graph_stats()["replays"] >= 8 and den.graph_stats()["failed"] == 0
    assert torch.equal(outs[I.CONSERVATIVE, 1], outs[I.AGGRESSIVE, 1])
    den.close()
