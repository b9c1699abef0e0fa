"""The operators around a block's Linears at the ends of their values and on every kernel by name: rows of any magnitude through the norms, infinite weights of an adapter, and
each tile and form of the products, which the probe names, beside rows and scratch that are no numbers.  References are those of test_gpu_block_operators.py, and so are the
tolerances; a result that is no number is refused wherever the reference has one."""
import numpy as np
import pytest

from test_gpu_block_operator_edges import FAR, far
from test_gpu_block_operators import HALF, adapted, adapter_case, f64, ffn, ffn_case, normed, rand, run_adapters
from test_gpu_block_operators import drf, forced, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def close(got, want, dtype, slack):
    """|got - want| <= half a step of the result + slack where the reference is finite, which no NaN and no infinity is; the reference's infinities and NaN elsewhere."""
    fine = np.isfinite(want)
    assert got.shape == want.shape and np.array_equal(got[~fine], want[~fine], equal_nan=True)
    slack = np.broadcast_to(slack, want.shape)
    bad = ~(np.abs(got[fine] - want[fine]) <= HALF[dtype] * np.abs(want[fine]) + slack[fine])
    assert not bad.any(), (int(bad.sum()), got[fine][bad][:4], want[fine][bad][:4])


# ---- magnitudes ---------------------------------------------------------------------------------------------

# A row's largest values.  Their squares pass fp32 from 1.8e19 on, sums of them over 1152 columns from 5.4e17, over 16384 from 1.4e17; squares vanish below 1e-22, the ones
# that hold 24 bits end at 1e-19.  (bf16 values below 1e-30 would themselves be rounded to fewer bits.)
MAGNITUDES = [1.0, 1e17, 3e17, 1e18, 1e19, 1e25, 1e32, 1e-12, 1e-17, 1e-19, 1e-21, 1e-23, 1e-30]


def rows_of_magnitudes(torch, rng, S, N, D, dtype):  # noqa: F811
    at = np.array(MAGNITUDES)[np.arange(S * N) % len(MAGNITUDES)].reshape(S, N, 1)
    v = rng.standard_normal((S, N, D)) + 0.5
    return torch.from_numpy((v / np.abs(v).max(-1, keepdims=True) * at).astype(np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()


@pytest.mark.parametrize("stream,branch", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("eps", [0.0, 1e-40, 1e-20, 1e-6])
@pytest.mark.parametrize("S,N,D", [(1, 13, 1152), (3, 800, 136), (3, 800, 1152), (2, 26, 2050), (1, 13, 16384), (1, 13, 3), (1, 26, 70)])
def test_norms_of_any_magnitude(torch, drf, stream, branch, kind, eps, S, N, D):  # noqa: F811
    """Rows of a wave, of a slot's staged modulation and of a workgroup, on both sides of the sum; every row beside others of other magnitudes.  The bound of a norm is
    relative to its deviation, so it is that of rows of ordinary size: a power of two taken out of a row costs nothing."""
    rng = np.random.default_rng(D + N)
    x, y = rows_of_magnitudes(torch, rng, S, N, D, stream), rows_of_magnitudes(torch, rng, S, N, D, branch)
    gain = rand(torch, rng, (D,), "f32", 0.3, 1.0)
    for t, dtype, got in ((x, stream, drf.residual_norm(x, before=kind, before_gain=gain, eps=eps)[1]),
                          (y, stream, drf.residual_norm(torch.zeros_like(x), y, after=kind, after_gain=gain, before=None, eps=eps)[0])):
        want, slack = normed(f64(t), kind, f64(gain), None, eps, 0 * f64(t))
        close(f64(got), want, dtype, slack + 2.0 ** -23 * np.abs(want))


def test_rows_without_a_norm_of_their_own(torch, drf):  # noqa: F811
    """Zeros (with an eps), an infinity, a NaN beside rows of the ends: each by the formula, the others as if alone."""
    rng = np.random.default_rng(8)
    for D in (72, 1152, 4100):
        x = rows_of_magnitudes(torch, rng, 1, 13, D, "f32")
        for eps in (1e-6, 1e-40):
            want = drf.residual_norm(x, before="rms", eps=eps)[1].clone()
            t = x.clone()
            t[0, 1], t[0, 4, 3], t[0, 9, D - 1] = 0.0, float("inf"), float("nan")
            got = drf.residual_norm(t, before="rms", eps=eps)[1]
            keep = torch.tensor([i not in (1, 4, 9) for i in range(13)], device="cuda")
            assert torch.equal(got[0, keep], want[0, keep])
            assert (got[0, 1] == 0).all() and torch.isnan(got[0, 9]).all() and torch.isnan(got[0, 4, 3]) and (got[0, 4, :3] == 0).all() and (got[0, 4, 4:] == 0).all()


def test_without_a_branch_its_arguments_are_not_looked_at(torch, drf):  # noqa: F811
    x, g = torch.randn(2, 5, 64, device="cuda"), torch.randn(64, device="cuda")
    want = drf.residual_norm(x)[1]
    assert torch.equal(drf.residual_norm(x, after="none", after_gain=g, y_scale=float("nan"), gate=torch.full((2, 64), float("nan"), device="cuda"))[1], want)
    assert torch.equal(drf.residual_norm(x, after="rms", after_bias=g)[1], want)


# ---- infinite weights of an adapter ---------------------------------------------------------------------------

# tiles of bf16, forms for few rows (8 to 13), the tile of fp32 (14): those that a product can take.  Gate and value need pairs of pieces in a wave (not 7, 13); ranks of B whose
# rows are no 16-byte pieces leave the largest tiles out; fp32 has four forms
STORE = {"bf16": list(range(14)), "f32": [8, 10, 11, 12, 14]}
GLU = {"bf16": [t for t in range(14) if t not in (7, 13)], "f32": STORE["f32"]}
ADAPT = {"bf16": STORE["bf16"], "f32": STORE["f32"]}
ADAPT_ODD = {"bf16": [t for t in range(14) if t not in (0, 1, 6, 7)], "f32": STORE["f32"]}
each = lambda kinds: [(d, t) for d in ("bf16", "f32") for t in kinds[d]]  # noqa: E731


def on(drf, forced, tile, kind, call):  # noqa: F811
    """The call's result, with its product of that kind held to the tile, on which it ran."""
    forced(tile)
    out = call()
    assert drf.probe_linear_route(kind) == tile
    return out


@pytest.mark.parametrize("R", [8, 24, 40, 5])
@pytest.mark.parametrize("S,N", [(2, 70), (6, 3), (1, 300)])
def test_infinite_weights_of_an_adapter(torch, drf, forced, R, S, N):  # noqa: F811
    """x A^T of whole numbers (which eight bits hold) and of zeros times an infinite weight: an infinity of its sign, or no number where it is zero."""
    rng = np.random.default_rng(R)
    D, O = 64, 72
    x = torch.from_numpy(rng.integers(-3, 4, (S, N, D)).astype(np.float32))
    w, a, b = torch.zeros(O, D), torch.zeros(2, R, D), torch.from_numpy(rng.integers(1, 5, (2, O, R)).astype(np.float32))
    a[:, torch.arange(R), torch.arange(R)] = 1.0                    # (x A^T: the first columns of x)
    a[1] *= 0.5
    b[0, 3, 2], b[0, 5, R - 1], b[1, 4, 0] = float("inf"), float("-inf"), float("inf")
    w[:, D - 1] = 1.0
    which = [j % 2 for j in range(S)]
    with np.errstate(invalid="ignore"):
        t = [x[j, :, :R].double().numpy() * (1.0, 0.5)[which[j]] for j in range(S)]
        want = np.stack([x[j, :, D - 1:].double().numpy() + sum(t[j][:, r:r + 1] * b[which[j], :, r].double().numpy()[None] for r in range(R)) for j in range(S)])
    for dtype in ("bf16", "f32"):
        args = [v.to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda() for v in (x, w, a, b)]
        for tile in (ADAPT_ODD if R % 8 else ADAPT)[dtype]:
            got = f64(on(drf, forced, tile, 2, lambda: run_adapters(torch, drf, *args, which, None, None)))
            assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[np.isinf(want)], want[np.isinf(want)]), (dtype, tile)
            fine = np.isfinite(want)
            close(got[fine], want[fine], dtype, 0.0)


def test_infinite_scales(torch, drf):  # noqa: F811
    """x A^T is infinite, and so is what finite and infinite weights of its sign make of it."""
    x, w, a = torch.ones(1, 20, 8, device="cuda"), torch.zeros(8, 8, device="cuda"), torch.ones(1, 8, 8, device="cuda")
    b = torch.full((1, 8, 8), 2.0, device="cuda")
    b[0, 3, 1] = float("inf")
    b[0, 5] = -1.0
    i, s = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((1,), float("inf"), device="cuda")
    want = torch.full((1, 20, 8), float("inf"), device="cuda")
    want[..., 5] = float("-inf")
    for t in (torch.float32, torch.bfloat16):
        assert torch.equal(drf.linear_adapters(x.to(t), w.to(t), a.to(t), b.to(t), i, None, s).float(), want)


# ---- every tile and form, by name -------------------------------------------------------------------------------

SHAPES = [(3, 70, 64, 136, 264), (5, 130, 200, 272, 300), (40, 9, 448, 152, 65), (1, 300, 72, 80, 72)]
LENS = lambda S, N: [(N, 0, 1, N // 2, N - 1)[j % 5] for j in range(S)]  # noqa: E731


def native(torch, drf, name, args, out):  # noqa: F811
    """The call with scratch that holds no number."""
    ops = drf._block_operators()
    call = getattr(ops, name)
    n = call(*args, None, None)
    scratch = torch.full((n // 2,), float("nan"), dtype=torch.bfloat16, device="cuda")
    drf._check(call(*args, out, scratch))
    return out


def poisoned(x, lens):
    y = x.clone()
    for j, n in enumerate(lens):
        y[j, n:] = float("nan")
    return y


def inside(got, want, slack, lens, dtype):
    for j, n in enumerate(lens):
        assert (got[j, n:] == 7).all()
        close(f64(got[j, :n]), want[j, :n], dtype, slack[j, :n])


@pytest.mark.parametrize("dtype,tile", each(STORE))
@pytest.mark.parametrize("S,N,D,F,O", SHAPES)
def test_gated_ffn_by_name(torch, drf, forced, dtype, tile, S, N, D, F, O):  # noqa: F811
    """Both products on the tile (or the first by choice, where it takes no gate and value), rows behind lengths and scratch are NaN: live rows are what they were."""
    rng = np.random.default_rng(N + D)
    x, w_in, w_out, b_in, b_out = ffn_case(torch, rng, S, N, D, F, O, dtype)
    want, slack = ffn(f64(x), f64(w_in), f64(w_out), f64(b_in), f64(b_out), "silu", dtype)
    lens = LENS(S, N)
    for n in (None, lens):
        t = None if n is None else torch.tensor(n, dtype=torch.int32, device="cuda")
        out = torch.full((S, N, O), 7.0, dtype=x.dtype, device="cuda")
        args = (x if n is None else poisoned(x, n), w_in, w_out, b_in, b_out, drf.GLU_SILU, t)
        got = on(drf, forced, tile, 0, lambda: native(torch, drf, "gated_ffn", args, out))
        assert tile not in GLU[dtype] or drf.probe_linear_route(1) == tile
        inside(got, want, slack, [N] * S if n is None else n, dtype)


@pytest.mark.parametrize("R,dtype,tile", [(R, *k) for R in (8, 40, 5) for k in each(ADAPT_ODD if R % 8 else ADAPT)])
@pytest.mark.parametrize("S,N,D,_,O", SHAPES)
def test_linear_adapters_by_name(torch, drf, forced, dtype, tile, R, S, N, D, _, O):  # noqa: F811
    rng = np.random.default_rng(N + D + R)
    x, w, a, b, _, bias, scales = adapter_case(torch, rng, S, N, D, O, R, 3, dtype)
    which = [(1, -1, 0, 2, 2)[j % 5] for j in range(S)]
    want, slack = adapted(f64(x), f64(w), f64(a), f64(b), which, f64(bias), f64(scales), dtype)
    i = torch.tensor(which, dtype=torch.int32, device="cuda")
    for n in (None, LENS(S, N)):
        t = None if n is None else torch.tensor(n, dtype=torch.int32, device="cuda")
        out = torch.full((S, N, O), 7.0, dtype=x.dtype, device="cuda")
        args = (x if n is None else poisoned(x, n), w, a, b, i, bias, scales, t)
        got = on(drf, forced, tile, 2, lambda: native(torch, drf, "linear_adapters", args, out))
        inside(got, want, slack, [N] * S if n is None else n, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,N,ss,ts", FAR)
def test_offsets_past_32_bits_by_name(torch, drf, forced, dtype, S, N, ss, ts):  # noqa: F811
    rng = np.random.default_rng(N)
    x, w_in, w_out, b_in, b_out = ffn_case(torch, rng, S, N, 136, 64, 136, dtype)
    _, w, a, b, which, bias, scales = adapter_case(torch, rng, S, N, 136, 136, 40, 3, dtype)
    block, low = ffn(f64(x), f64(w_in), f64(w_out), f64(b_in), f64(b_out), "silu", dtype), adapted(f64(x), f64(w), f64(a), f64(b), which, f64(bias), f64(scales), dtype)
    wide, out = far(torch, x.shape, (ss, ts), x.dtype).copy_(x), far(torch, x.shape, (ss, ts), x.dtype)
    for tile in STORE[dtype]:
        out.fill_(7.0)
        close(f64(on(drf, forced, tile, 0, lambda: drf.gated_ffn(wide, w_in, w_out, b_in, b_out, out=out))), block[0], dtype, block[1])
        out.fill_(7.0)
        close(f64(on(drf, forced, tile, 2, lambda: run_adapters(torch, drf, wide, w, a, b, which, bias, scales, out=out))), low[0], dtype, low[1])
    del wide, out
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def test_the_probe_names_what_ran(torch, drf, forced):  # noqa: F811
    """A number that a product cannot take leaves the choice to the model, and the probe says so."""
    rng = np.random.default_rng(1)
    c = ffn_case(torch, rng, 1, 300, 72, 80, 72, "f32")
    forced(-1)
    drf.gated_ffn(*c)
    chosen = [drf.probe_linear_route(k) for k in (0, 1)]
    assert all(k in STORE["f32"] for k in chosen)
    for tile in (0, 7, 9, 13):
        forced(tile)
        drf.gated_ffn(*c)
        assert [drf.probe_linear_route(k) for k in (0, 1)] == chosen
    assert drf.probe_linear_route(3) == drf.probe_linear_route(-1) == -1
