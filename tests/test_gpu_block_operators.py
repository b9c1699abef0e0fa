"""The operators around a block's Linears against their definitions in float64 (numpy), at the sizes, layouts, lengths and values where they can go wrong.

Tolerances.  A rounding is off by at most half a step, 2^-8 of the value in bf16 and 2^-24 in fp32 (u below).
  sums: n terms in fp32, in any order, are off by (n + 8) u of the sum of their magnitudes at most; in fp32 each product is rounded too: twice that.
  norms: a lane adds up to 32 columns, then some 9 levels: a mean is off by 48 u of the mean magnitude, a variance by as much of itself, squares and root by
      4 u; with n the normed value and m the mean magnitude over the deviation: 48 u m + 28 u |n| + 48 u, below 2^-18 (m + 1 + |n|).
  activations: exponent and reciprocal to 2^-20, absolute (|a|^2 e^-|a| and the like are below one) and of the value; their slope is below 1.13.
  feed-forward, bf16: the product of act and value is rounded once to bf16, as the operand of the second product.
  adapters, bf16: x A^T is taken to 16 bits, 2^-16 of it lost."""
import numpy as np
import pytest

from paper_2603_25872_amd import drf as D_

pytestmark = pytest.mark.gpu
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available()
    return t


@pytest.fixture(scope="module")
def drf():
    D_.lib()
    return D_


def dtype_of(torch, name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def f64(t):
    return t.detach().double().cpu().numpy()


def rand(torch, rng, shape, dtype="f32", scale=1.0, offset=0.0):
    return torch.from_numpy((rng.standard_normal(shape) * scale + offset).astype(np.float32)).to(dtype_of(torch, dtype)).cuda()


def laid(torch, x, layout):
    """x [slots, tokens, columns] in one of the memory layouts that a caller may have."""
    S, N, D = x.shape
    if layout == "rows":                                            # a column range of wider rows
        y = torch.empty(S, N, D + 24, dtype=x.dtype, device="cuda")[..., 8:8 + D]
    elif layout == "odd":                                           # nothing is aligned to 16 bytes
        y = torch.empty(S * N * (D + 3) + 1, dtype=x.dtype, device="cuda")[1:].view(S, N, D + 3)[..., :D]
    elif layout == "tokens":                                        # token by token, the slots beside one another
        y = torch.empty(N, S, D, dtype=x.dtype, device="cuda").transpose(0, 1)
    else:
        y = torch.empty(S, N, D, dtype=x.dtype, device="cuda")
    return y.copy_(x)


def check(got, want, dtype, slack):
    """|got - want| <= half a step of the result + slack, everywhere; NaN and infinities where the reference has them."""
    got = f64(got)
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine], equal_nan=True)
    off = np.abs(got - np.where(fine, want, got)) - (HALF[dtype] * np.abs(np.where(fine, want, 0.0)) + slack)
    assert not (off[fine] > 0).any(), (int((off[fine] > 0).sum()), float(off[fine].max()))


# ---- residual stream and norms ---------------------------------------------------------------------------


def normed(x, kind, gain, bias, eps, err):
    """The norm of rows and how far it may be off where x is off by err."""
    if kind == "none":
        return x, err
    c = x - x.mean(-1, keepdims=True) if kind == "layer" else x
    dev = np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    n = c / dev
    m = np.abs(x).mean(-1, keepdims=True) / dev
    g = 1.0 if gain is None else np.abs(gain)
    off = (2.0 ** -18 * (m + 1 + np.abs(n)) + (err + np.max(err, -1, keepdims=True) * (1 + np.abs(n))) / dev) * g
    n = n * (1 if gain is None else gain) + (0 if bias is None else bias)
    return n, off + 2 * U * np.abs(n)


def residual(x, y, a):
    """(z, its slack, h, its slack) in float64 of drf.residual_norm's arguments."""
    mod = lambda t: None if t is None else (t if t.ndim == 3 else t[:, None])  # noqa: E731
    z, off = a["x_scale"] * x, U * np.abs(x * a["x_scale"])
    if y is not None:
        n, err = normed(y, a["after"], a["after_gain"], a["after_bias"], a["eps"], 0 * y)
        g = a["y_scale"] * (1.0 if a["gate"] is None else mod(a["gate"]))
        z, off = z + g * n, off + np.abs(g) * (err + 2 * U * np.abs(n))
    off = off + 2 * U * np.abs(z)
    h, err = normed(z, a["before"], a["before_gain"], a["before_bias"], a["eps"], off)
    s = 1.0 if a["scale"] is None else 1.0 + mod(a["scale"])
    h, err = h * s, err * np.abs(s) + 3 * U * np.abs(h * s)
    if a["shift"] is not None:
        h = h + mod(a["shift"])
    return z, off, h, err + 2 * U * np.abs(h)


def residual_case(torch, rng, S, N, D, stream, branch, after, before, layout, per_token=False, offset=0.0):
    x = laid(torch, rand(torch, rng, (S, N, D), stream, 3.0, offset), layout)
    y = laid(torch, rand(torch, rng, (S, N, D), branch, 1.0, offset), layout)
    rows = rand(torch, rng, (S, N, 6 * D) if per_token else (S, 6 * D), "f32", 0.5)
    a = dict(gate=rows[..., :D], shift=rows[..., D:2 * D], scale=rows[..., 3 * D:4 * D], after=after, before=before, x_scale=0.75, y_scale=-1.5, eps=1e-5)
    vec = lambda: rand(torch, rng, (D,), "f32", 0.3, 1.0)  # noqa: E731
    a.update(after_gain=None if after == "none" else vec(), after_bias=vec() if after == "layer" else None,
             before_gain=None if before == "none" else vec(), before_bias=vec() if before == "layer" else None)
    return x, y, a, {k: f64(v) if hasattr(v, "device") else v for k, v in a.items()}


TYPES = [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")]
NORMS = ["none", "rms", "layer"]


@pytest.mark.parametrize("stream,branch", TYPES)
@pytest.mark.parametrize("after", NORMS)
@pytest.mark.parametrize("before", NORMS)
@pytest.mark.parametrize("layout,D", [("plain", 72), ("rows", 384), ("odd", 130), ("tokens", 1152)])
def test_residual_norm(torch, drf, stream, branch, after, before, layout, D):
    rng = np.random.default_rng(D)
    x, y, a, r = residual_case(torch, rng, 3, 7, D, stream, branch, after, before, layout)
    z, h = drf.residual_norm(x, y, **a)
    zz, ez, hh, eh = residual(f64(x), f64(y), r)
    assert z.dtype == x.dtype and h.dtype == y.dtype
    check(z, zz, stream, ez)
    check(h, hh, branch, eh)


@pytest.mark.parametrize("stream,branch", TYPES)
@pytest.mark.parametrize("D", [1, 2, 3, 8, 63, 64, 65, 500, 512, 514, 520, 1024, 1536, 1544, 2048, 2049, 2050, 2056, 4096, 4100, 6000, 8192, 8200, 12345, 16384])
def test_residual_norm_widths(torch, drf, stream, branch, D):
    """Every number of columns a lane holds and of waves a row takes, per-token modulations, one token and several."""
    rng = np.random.default_rng(D)
    for S, N, after, before in ((1, 1, "none", "layer"), (2, 5, "rms", "rms"), (2, 3, "layer", "layer")):
        x, y, a, r = residual_case(torch, rng, S, N, D, stream, branch, after, before, "plain", per_token=N == 5)
        if D == 1 and before == "layer":                            # a deviation of nothing: rounding alone would decide the value
            a["before"] = r["before"] = "rms"
            a["before_bias"] = r["before_bias"] = None
        z, h = drf.residual_norm(x, y, **a)
        zz, ez, hh, eh = residual(f64(x), f64(y), r)
        check(z, zz, stream, ez)
        check(h, hh, branch, eh)


@pytest.mark.parametrize("stream,branch", TYPES)
@pytest.mark.parametrize("N,D", [(1024, 768), (4099, 40), (37, 4096), (2500, 100)])
def test_residual_norm_of_many_rows(torch, drf, stream, branch, N, D):
    """More rows than a workgroup takes at once, and more than a launch has workgroups of one row."""
    rng = np.random.default_rng(N)
    x, y, a, r = residual_case(torch, rng, 3, N, D, stream, branch, "rms", "layer", "plain")
    z, h = drf.residual_norm(x, y, **a)
    zz, ez, hh, eh = residual(f64(x), f64(y), r)
    check(z, zz, stream, ez)
    check(h, hh, branch, eh)


@pytest.mark.parametrize("stream,branch", TYPES)
@pytest.mark.parametrize("D", [130, 384, 3000])
def test_residual_norm_parts_of_it(torch, drf, stream, branch, D):
    """Without a branch, without a norm of the sum, in place, without parameters."""
    rng = np.random.default_rng(D)
    x, y, a, r = residual_case(torch, rng, 2, 9, D, stream, branch, "rms", "layer", "plain")
    zz, ez, hh, eh = residual(f64(x), f64(y), r)
    z, h = drf.residual_norm(x, y, **dict(a, before=None, before_gain=None, before_bias=None))
    assert h is None
    check(z, zz, stream, ez)
    x2, y2 = x.clone(), y.clone()
    z, h = drf.residual_norm(x2, y2, **a, out=x2, h_out=y2)
    assert z is x2 and h is y2
    check(z, zz, stream, ez)
    check(h, hh, branch, eh)
    z, h = drf.residual_norm(x, **a)
    _, _, hh, eh = residual(f64(x), None, r)
    assert z is x and h.dtype == x.dtype
    check(h, hh, stream, eh)
    z, h = drf.residual_norm(x, h_out=y2, **a)                      # a stream in fp32 for a branch in bf16
    check(h, hh, branch, eh)
    z, h = drf.residual_norm(x, y)
    zz, ez, hh, eh = residual(f64(x), f64(y), dict(dict.fromkeys(r), x_scale=1.0, y_scale=1.0, after="none", before="layer", eps=1e-6))
    check(z, zz, stream, ez)
    check(h, hh, branch, eh)


@pytest.mark.parametrize("stream,branch", TYPES)
@pytest.mark.parametrize("N,D", [(11, 72), (11, 131), (11, 2500), (600, 72), (600, 131), (500, 1153)])
def test_residual_norm_lengths(torch, drf, stream, branch, N, D):
    """Rows behind a slot's length are neither read (they are NaN) nor written; lengths of none, one, all, fewer than none and more than all."""
    rng = np.random.default_rng(D)
    S = 6
    x, y, a, r = residual_case(torch, rng, S, N, D, stream, branch, "layer", "rms", "plain")
    zz, ez, hh, eh = residual(f64(x), f64(y), r)
    lens = [0, 1, N, -5, N + 100, N // 2 + 1]
    for j, n in enumerate(lens):
        n = min(max(n, 0), N)
        x[j, n:] = float("nan")
        y[j, n:] = float("nan")
    z, h = torch.full_like(x, 7.0), torch.full_like(y, 7.0)
    t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    drf.residual_norm(x, y, **a, lens=t, out=z, h_out=h)
    for j, n in enumerate(lens):
        n = min(max(n, 0), N)
        assert (z[j, n:] == 7).all() and (h[j, n:] == 7).all()
        check(z[j, :n], zz[j, :n], stream, ez[j, :n])
        check(h[j, :n], hh[j, :n], branch, eh[j, :n])
    z, h = drf.residual_norm(x, y, **a, lens=t)
    assert (h[0] == 0).all() and torch.isnan(z[0]).all()


def test_residual_norm_values(torch, drf):
    """A row of equal values, of zeros, with a mean far from zero, with an infinity: each by its formula, and its neighbours untouched by it."""
    D = 256
    x = torch.zeros(1, 5, D, device="cuda")
    x[0, 1] = 3.5
    x[0, 2] = 1000 + torch.arange(D, device="cuda") % 2                 # exact in fp32: mean 1000.5, deviation 0.5
    x[0, 3, 7] = float("inf")
    x[0, 4] = torch.arange(D, device="cuda")
    for eps in (1e-6, 1e-50, 0.25):
        h = f64(drf.residual_norm(x, before="layer", eps=eps)[1])
        assert (h[0, :2] == 0).all() and np.isnan(h[0, 3]).all()
        assert np.abs(h[0, 2] - (x[0, 2].cpu().numpy() - 1000.5) / np.sqrt(0.25 + eps)).max() < 2.0 ** -20
        want = (np.arange(D) - 127.5) / np.sqrt((D * D - 1) / 12 + eps)
        assert np.abs(h[0, 4] - want).max() < 2.0 ** -19
        r = f64(drf.residual_norm(x, before="rms", eps=eps)[1])
        assert (r[0, 0] == 0).all() and np.isnan(r[0, 3, 7]) and (r[0, 3, :7] == 0).all()


# ---- gated feed-forward ----------------------------------------------------------------------------------


def act_of(a, act):
    return a / (1 + np.exp(-a)) if act == "silu" else 0.5 * a * (1 + np.tanh(np.sqrt(2 / np.pi) * (a + 0.044715 * a ** 3)))


def ffn(x, w_in, w_out, b_in, b_out, act, dtype):
    """The block in float64, and its slack."""
    F, D = w_out.shape[1], x.shape[-1]
    twice = 1 if dtype == "bf16" else 2
    with np.errstate(over="ignore"):
        u = x @ w_in.T + (0 if b_in is None else b_in)
        eu = twice * (D + 8) * U * (np.abs(x) @ np.abs(w_in).T) + 2 * U * np.abs(u)
        g, v, eg, ev = u[..., :F], u[..., F:], eu[..., :F], eu[..., F:]
        s = act_of(g, act)
    es = 1.13 * eg + 2.0 ** -20 * (1 + np.abs(s))
    p = s * v
    ep = es * (np.abs(v) + ev) + np.abs(s) * ev + HALF[dtype] * np.abs(p) + 2.0 ** -133
    y = p @ w_out.T + (0 if b_out is None else b_out)
    return y, ep @ np.abs(w_out).T + twice * (F + 8) * U * (np.abs(p) @ np.abs(w_out).T) + 2 * U * np.abs(y)


def ffn_case(torch, rng, S, N, D, F, O, dtype, layout="plain", bias=True):
    x = laid(torch, rand(torch, rng, (S, N, D), dtype), layout)
    w_in, w_out = rand(torch, rng, (2 * F, D), dtype, D ** -0.5), rand(torch, rng, (O, F), dtype, F ** -0.5)
    return x, w_in, w_out, rand(torch, rng, (2 * F,), "f32", 0.5) if bias else None, rand(torch, rng, (O,), "f32", 0.5) if bias else None


def opt(t):
    return None if t is None else f64(t)


FFN = [(1, 1, 8, 8, 8), (1, 1, 1152, 512, 384), (3, 1, 64, 72, 40), (2, 33, 72, 104, 72), (1, 64, 128, 128, 128), (2, 100, 200, 136, 201), (5, 77, 384, 264, 130),
       (1, 300, 1000, 320, 96), (1, 257, 520, 1032, 264), (70, 1, 48, 24, 7), (3, 129, 64, 32, 1), (1, 1500, 96, 160, 96)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("S,N,D,F,O", FFN)
def test_gated_ffn(torch, drf, dtype, act, S, N, D, F, O):
    rng = np.random.default_rng(N + D)
    for layout, bias in (("plain", True), ("rows", False), ("tokens", True)):
        x, w_in, w_out, b_in, b_out = ffn_case(torch, rng, S, N, D, F, O, dtype, layout, bias)
        got = drf.gated_ffn(x, w_in, w_out, b_in, b_out, act)
        assert got.dtype == x.dtype and got.shape == (S, N, O)
        want, slack = ffn(f64(x), f64(w_in), f64(w_out), opt(b_in), opt(b_out), act, dtype)
        check(got, want, dtype, slack)


@pytest.mark.parametrize("S,N,D,F,O", [(1, 1, 1, 1, 1), (2, 37, 61, 47, 35), (1, 130, 250, 694, 250), (3, 70, 17, 33, 65)])
def test_gated_ffn_odd_fp32(torch, drf, S, N, D, F, O):
    """Widths that no vector divides, and rows that no vector's address is."""
    rng = np.random.default_rng(D)
    for layout in ("plain", "odd"):
        x, w_in, w_out, b_in, b_out = ffn_case(torch, rng, S, N, D, F, O, "f32", layout)
        want, slack = ffn(f64(x), f64(w_in), f64(w_out), f64(b_in), f64(b_out), "silu", "f32")
        check(drf.gated_ffn(x, w_in, w_out, b_in, b_out), want, "f32", slack)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,F,O", [(70, 72, 40, 72), (300, 256, 128, 256), (3, 64, 64, 65)])
@pytest.mark.parametrize("layout", ["plain", "odd"])
def test_gated_ffn_lengths(torch, drf, dtype, N, D, F, O, layout):
    """Rows behind a slot's length (NaN here) reach nothing and are left as they were."""
    rng = np.random.default_rng(N)
    x, w_in, w_out, b_in, b_out = ffn_case(torch, rng, 6, N, D, F, O, dtype)
    want, slack = ffn(f64(x), f64(w_in), f64(w_out), f64(b_in), f64(b_out), "silu", dtype)
    lens = [0, 1, N, -1, N + 9, N // 2]
    for j, n in enumerate(lens):
        x[j, max(n, 0):] = float("nan")
    out = laid(torch, torch.full((6, N, O), 7.0, dtype=x.dtype, device="cuda"), layout)
    drf.gated_ffn(x, w_in, w_out, b_in, b_out, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), out=out)
    for j, n in enumerate(lens):
        n = min(max(n, 0), N)
        assert (out[j, n:] == 7).all()
        check(out[j, :n], want[j, :n], dtype, slack[j, :n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [5, 200])
def test_gated_ffn_rows_are_their_own(torch, drf, dtype, N):
    """A row that is no number is nothing to the others; one row for all slots and tokens; gates far from zero on both sides."""
    rng = np.random.default_rng(N)
    x, w_in, w_out, b_in, b_out = ffn_case(torch, rng, 2, N, 136, 72, 136, dtype)
    want = drf.gated_ffn(x, w_in, w_out, b_in, b_out)
    x[1, 3, 5] = float("nan")
    x[0, 2, 7] = float("inf")
    got = drf.gated_ffn(x, w_in, w_out, b_in, b_out)
    assert torch.isnan(got[1, 3]).all() and not torch.isfinite(got[0, 2]).any()
    keep = torch.ones(2, N, dtype=torch.bool, device="cuda")
    keep[1, 3] = keep[0, 2] = False
    assert torch.equal(got[keep], want[keep])
    one = rand(torch, rng, (1, 1, 136), dtype)
    got = drf.gated_ffn(one.expand(3, N, 136), w_in, w_out, b_in, b_out)
    want, slack = ffn(f64(one), f64(w_in), f64(w_out), f64(b_in), f64(b_out), "silu", dtype)
    check(got, np.broadcast_to(want, got.shape), dtype, slack)
    big = rand(torch, rng, (1, N, 136), dtype, 60.0)
    for act in ("silu", "gelu"):
        want, slack = ffn(f64(big), f64(w_in), f64(w_out), f64(b_in), f64(b_out), act, dtype)
        check(drf.gated_ffn(big, w_in, w_out, b_in, b_out, act), want, dtype, slack)


# ---- low-rank adapters -----------------------------------------------------------------------------------


def adapted(x, w, a, b, which, bias, scales, dtype):
    D, R = x.shape[-1], a.shape[1]
    twice = 1 if dtype == "bf16" else 2
    y = x @ w.T
    slack = twice * (D + R + 8) * U * (np.abs(x) @ np.abs(w).T)
    for j, i in enumerate(which):
        if 0 <= i < a.shape[0]:
            s = 1.0 if scales is None else scales[i]
            t = s * (x[j] @ a[i].T)
            et = twice * (D + 8) * U * abs(s) * (np.abs(x[j]) @ np.abs(a[i]).T) + (2.0 ** -16 if dtype == "bf16" else 2 * U) * np.abs(t) + 2.0 ** -126
            y[j] += t @ b[i].T
            slack[j] += et @ np.abs(b[i]).T + twice * (D + R + 8) * U * (np.abs(t) @ np.abs(b[i]).T)
    y = y + (0 if bias is None else bias)
    return y, slack + 2 * U * np.abs(y)


def adapter_case(torch, rng, S, N, D, O, R, n, dtype, layout="plain", bias=True):
    x = laid(torch, rand(torch, rng, (S, N, D), dtype), layout)
    w, a, b = rand(torch, rng, (O, D), dtype, D ** -0.5), rand(torch, rng, (n, R, D), dtype, D ** -0.5), rand(torch, rng, (n, O, R), dtype, R ** -0.5)
    which = rng.integers(-1, n, S).astype(np.int32)
    return x, w, a, b, which, rand(torch, rng, (O,), "f32", 0.5) if bias else None, rand(torch, rng, (n,), "f32", 0.5, 1.0) if bias else None


def run_adapters(torch, drf, x, w, a, b, which, bias, scales, **kw):
    return drf.linear_adapters(x, w, a, b, torch.tensor(which, dtype=torch.int32, device="cuda"), bias, scales, **kw)


ADAPT = [(1, 1, 8, 8, 1, 1), (64, 1, 128, 200, 16, 9), (3, 1, 1152, 136, 8, 3), (5, 33, 72, 104, 5, 2), (2, 64, 128, 128, 32, 2), (7, 77, 200, 130, 24, 7), (3, 100, 64, 65, 17, 3),
         (1, 300, 520, 264, 64, 1), (4, 130, 96, 72, 128, 4), (2, 40, 48, 40, 256, 2), (40, 3, 64, 72, 12, 40), (2, 700, 136, 288, 33, 5), (130, 2, 40, 24, 4, 130)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,N,D,O,R,n", ADAPT)
def test_linear_adapters(torch, drf, dtype, S, N, D, O, R, n):
    rng = np.random.default_rng(N + D + R)
    for layout, bias in (("plain", True), ("rows", False), ("tokens", True)):
        c = adapter_case(torch, rng, S, N, D, O, R, n, dtype, layout, bias)
        got = run_adapters(torch, drf, *c)
        assert got.dtype == c[0].dtype and got.shape == (S, N, O)
        want, slack = adapted(*[f64(v) for v in c[:4]], c[4], opt(c[5]), opt(c[6]), dtype)
        check(got, want, dtype, slack)


@pytest.mark.parametrize("S,N,D,O,R,n", [(1, 1, 1, 1, 1, 1), (3, 37, 61, 47, 7, 2), (2, 130, 250, 694, 50, 3)])
def test_linear_adapters_odd_fp32(torch, drf, S, N, D, O, R, n):
    rng = np.random.default_rng(D)
    for layout in ("plain", "odd"):
        c = adapter_case(torch, rng, S, N, D, O, R, n, "f32", layout)
        want, slack = adapted(*[f64(v) for v in c[:4]], c[4], f64(c[5]), f64(c[6]), "f32")
        check(run_adapters(torch, drf, *c), want, "f32", slack)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 5, 70, 200])
def test_linear_adapters_of_some_slots(torch, drf, dtype, N):
    """All slots without an adapter, indices outside of the adapters, none at all, every slot the same one; lengths."""
    rng = np.random.default_rng(N)
    S = 9
    x, w, a, b, _, bias, scales = adapter_case(torch, rng, S, N, 104, 72, 12, 3, dtype)
    plain = run_adapters(torch, drf, x, w, a[:0], b[:0], [0] * S, bias, None)
    for which in ([-1] * S, [3] * S, [-2 ** 31, 2 ** 31 - 1, 3, -7, 99, -1, 5, 1000, 4]):
        assert torch.equal(run_adapters(torch, drf, x, w, a, b, which, bias, scales), plain)
    for which in ([1] * S, [0, 0, 1, 1, -1, 2, 2, 7, 0]):
        want, slack = adapted(f64(x), f64(w), f64(a), f64(b), which, f64(bias), f64(scales), dtype)
        check(run_adapters(torch, drf, x, w, a, b, which, bias, scales), want, dtype, slack)
        lens = [0, 1, N, -4, N + 3, N // 2, N, N // 3, 1]
        y = x.clone()
        for j, k in enumerate(lens):
            y[j, max(k, 0):] = float("nan")
        out = torch.full_like(plain, 7.0)
        run_adapters(torch, drf, y, w, a, b, which, bias, scales, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), out=out)
        for j, k in enumerate(lens):
            k = min(max(k, 0), N)
            assert (out[j, k:] == 7).all()
            check(out[j, :k], want[j, :k], dtype, slack[j, :k])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,N,R", [(12, 1, 8), (12, 1, 40), (12, 7, 16), (4, 100, 24), (3, 300, 64)])
def test_adapters_are_their_slots_own(torch, drf, dtype, S, N, R):
    """An adapter whose weights or scale are infinite or no number, and rows that are, reach their own slots and rows alone, bit for bit."""
    rng = np.random.default_rng(R)
    x, w, a, b, _, bias, scales = adapter_case(torch, rng, S, N, 72, 136, R, 3, dtype)
    which = [j % 3 - (j % 7 == 5) for j in range(S)]
    want = run_adapters(torch, drf, x, w, a, b, which, bias, scales)
    others = torch.tensor([i != 1 for i in which], device="cuda")
    for bad in (float("inf"), float("nan"), 3.3e38):
        for k in range(3):
            t = [a.clone(), b.clone(), scales.clone()]
            t[k][1] = bad
            got = run_adapters(torch, drf, x, w, t[0], t[1], which, bias, t[2])
            assert torch.equal(got[others], want[others])
            assert bad == 3.3e38 or not torch.isfinite(got[~others]).any()
    y = x.clone()
    y[1, 0, 3] = float("nan")
    y[2, N - 1, 3] = float("inf")
    got = run_adapters(torch, drf, y, w, a, b, which, bias, scales)
    assert torch.isnan(got[1, 0]).all() and not torch.isfinite(got[2, N - 1]).any()
    keep = torch.ones(S, N, dtype=torch.bool, device="cuda")
    keep[1, 0] = keep[2, N - 1] = False
    assert torch.equal(got[keep], want[keep])


# ---- as they are called ------------------------------------------------------------------------------------


def block(torch, drf, x, p, which, lens=None):
    """One block from public operators: adaLN, q | k | v with adapters, norms and rotation, attention over chosen blocks, projection with adapters, gated feed-forward."""
    S, N, D = x.shape
    H, d = p["heads"], D // p["heads"]
    m = [p["mod"][:, i * D:(i + 1) * D] for i in range(6)]
    _, h = drf.residual_norm(x, h_out=torch.zeros(S, N, D, dtype=p["qkv"].dtype, device="cuda"), shift=m[0], scale=m[1], lens=lens)
    qkv = drf.linear_adapters(h, p["qkv"], p["qkv_a"], p["qkv_b"], which, scales=p["scales"], lens=lens).view(S, N, 3 * H, d)
    q, k, v = qkv.split(H, dim=2)
    q, k = drf.qk_norm_rope(q, k, "rms", drf.rope_config((d // 2, d // 2), (1, 8)), lens=lens, q_out=q, k_out=k)
    o = drf.block_attention(q, k, v, drf.block_select(q, k, 32, 32, 2, q_lens=lens, kv_lens=lens), 32, 32, q_lens=lens, kv_lens=lens).reshape(S, N, D)
    y = drf.linear_adapters(o, p["proj"], p["proj_a"], p["proj_b"], which, lens=lens)
    x, h = drf.residual_norm(x, y, gate=m[2], after="rms", after_gain=p["gain"], shift=m[3], scale=m[4], lens=lens)
    y = drf.gated_ffn(h, p["w_in"], p["w_out"], act="silu", lens=lens)
    return drf.residual_norm(x, y, gate=m[5], after="rms", before=None, lens=lens)[0]


def block_parameters(torch, rng, S, D, H, F, R, n, dtype):
    t = lambda shape, scale: rand(torch, rng, shape, dtype, scale)  # noqa: E731
    return dict(heads=H, mod=rand(torch, rng, (S, 6 * D), "f32", 0.5), qkv=t((3 * D, D), D ** -0.5), qkv_a=t((n, R, D), D ** -0.5), qkv_b=t((n, 3 * D, R), R ** -0.5),
                proj=t((D, D), D ** -0.5), proj_a=t((n, R, D), D ** -0.5), proj_b=t((n, D, R), R ** -0.5), scales=rand(torch, rng, (n,), "f32", 0.3, 1.0),
                gain=rand(torch, rng, (D,), "f32", 0.2, 1.0), w_in=t((2 * F, D), D ** -0.5), w_out=t((D, F), F ** -0.5))


def plain_block(x, p, which):
    """The same in float64, one slot of its own length at a time; x [tokens, columns], m the slot's modulation rows."""
    def one(x, m, i):
        N, D = x.shape
        H, d = p["heads"], D // p["heads"]
        ln = lambda z: (z - z.mean(-1, keepdims=True)) / np.sqrt(z.var(-1, keepdims=True) + 1e-6)  # noqa: E731
        rms = lambda z: z / np.sqrt((z * z).mean(-1, keepdims=True) + 1e-6)  # noqa: E731
        low = lambda z, n, s: z @ p[n].T + (0 if i < 0 else (p["scales"][i] if s else 1) * (z @ p[n + "_a"][i].T) @ p[n + "_b"][i].T)  # noqa: E731
        q, k, v = (low(ln(x) * (1 + m[1]) + m[0], "qkv", True).reshape(N, 3, H, d)[:, j] for j in range(3))
        q, k = rms(q), rms(k)
        n = np.arange(N)
        for pos, at in ((n // 8 * 8 // 8, 0), (n % 8, d // 2)):
            for f in range(d // 4):
                c, s = np.cos(pos * 1e4 ** (-4.0 * f / d))[:, None], np.sin(pos * 1e4 ** (-4.0 * f / d))[:, None]
                for t in (q, k):
                    u, w = t[..., at + 2 * f].copy(), t[..., at + 2 * f + 1].copy()
                    t[..., at + 2 * f], t[..., at + 2 * f + 1] = u * c - w * s, u * s + w * c
        o = np.zeros((N, H, d))
        for h in range(H):
            e = np.exp(q[:, h] @ k[:, h].T * d ** -0.5)
            o[:, h] = e / e.sum(-1, keepdims=True) @ v[:, h]
        x = x + m[2] * rms(low(o.reshape(N, D), "proj", False)) * p["gain"]
        u = (ln(x) * (1 + m[4]) + m[3]) @ p["w_in"].T
        F = u.shape[1] // 2
        return x + m[5] * rms((act_of(u[:, :F], "silu") * u[:, F:]) @ p["w_out"].T)
    D = x[0].shape[-1]
    return [one(x[j], p["mod"][j].reshape(6, D), which[j]) for j in range(len(x))]


@pytest.mark.parametrize("dtype,tol", [("f32", 2e-5), ("bf16", 5e-2)])
def test_a_block_of_operators(torch, drf, dtype, tol):
    """A whole block (two key blocks of two: every key), slots of uneven length, against float64.  Tolerance: some 12 rounded steps between norms, each off by at most a few
    half steps of its largest values (fp32: 2^-24 times the square root of some thousand terms), relative to the largest value."""
    rng = np.random.default_rng(0)
    S, N, D, H, F, R, n = 4, 64, 128, 4, 192, 8, 3
    p = block_parameters(torch, rng, S, D, H, F, R, n, dtype)
    x = rand(torch, rng, (S, N, D))
    which, lens = [2, -1, 0, 1], [64, 33, 1, 50]
    got = f64(block(torch, drf, x, p, torch.tensor(which, dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda")))
    xs = f64(x)
    want = plain_block([xs[j, :k] for j, k in enumerate(lens)], {k: v if k == "heads" else f64(v) for k, v in p.items()}, which)
    for j, k in enumerate(lens):
        assert np.abs(got[j, :k] - want[j]).max() <= tol * np.abs(want[j]).max()
        assert np.array_equal(got[j, k:], xs[j, k:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_block_captured_and_replayed(torch, drf, dtype):
    """Recorded into a graph beside eager calls on other data; every replay gives the eager bits, also after the inputs changed in place."""
    rng = np.random.default_rng(1)
    p = block_parameters(torch, rng, 4, 128, 4, 192, 8, 3, dtype)
    xs = [rand(torch, rng, (4, 64, 128)) for _ in range(2)]
    which = [torch.tensor(w, dtype=torch.int32, device="cuda") for w in ([2, -1, 0, 1], [1, 1, -1, 2])]
    want = [block(torch, drf, x, p, w) for x, w in zip(xs, which)]
    x, w = xs[0].clone(), which[0].clone()
    torch.cuda.synchronize()
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block(torch, drf, x, p, w)
    with torch.cuda.graph(other):
        out2 = block(torch, drf, xs[1], p, which[1])
    for it in range(4):
        x.copy_(xs[it % 2])
        w.copy_(which[it % 2])
        out.fill_(float("nan"))
        graph.replay()
        other.replay()
        assert torch.equal(block(torch, drf, xs[1], p, which[1]), want[1])
        torch.cuda.synchronize()
        assert torch.equal(out, want[it % 2]) and torch.equal(out2, want[1]), it


def test_on_streams_of_their_own(torch, drf):
    """Calls on two streams at once give what one stream gives."""
    rng = np.random.default_rng(2)
    p = block_parameters(torch, rng, 8, 256, 4, 512, 16, 3, "bf16")
    x = rand(torch, rng, (8, 64, 256))
    w = torch.tensor([2, -1, 0, 1, 0, 0, 1, 2], dtype=torch.int32, device="cuda")
    want = block(torch, drf, x, p, w)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for _ in range(6):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(block(torch, drf, x, p, w))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_no_gradient_is_recorded(torch, drf):
    x = torch.randn(1, 4, 64, device="cuda", requires_grad=True)
    w = torch.randn(128, 64, device="cuda", requires_grad=True)
    lens, which = torch.tensor([3], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    outs = [*drf.residual_norm(x, x.detach() + 1, lens=lens), *drf.residual_norm(x, x.detach() + 1), drf.gated_ffn(x, w, w.detach()[:64].contiguous()),
            drf.linear_adapters(x, w, w[None, :2].contiguous(), w[None, :, :2].contiguous(), which)]
    assert not any(o.requires_grad for o in outs)


def test_bad_tensors_are_refused(torch, drf):
    x = torch.zeros(2, 4, 64, device="cuda")
    y, w, i = torch.zeros_like(x), torch.zeros(128, 64, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    a, b, v = w[None, :2].contiguous(), w[None, :, :2].contiguous(), torch.zeros(64, device="cuda")
    w_out = torch.zeros(64, 64, device="cuda")
    for call in (lambda: drf.residual_norm(x, y[:, :3]), lambda: drf.residual_norm(x[0], y[0]), lambda: drf.residual_norm(x, y.cpu()), lambda: drf.residual_norm(x.half(), y),
                 lambda: drf.residual_norm(x, y, gate=v), lambda: drf.residual_norm(x, y, shift=y[:, 0].half()), lambda: drf.residual_norm(x, y, before_gain=v[:63]),
                 lambda: drf.residual_norm(x, y, out=y.bfloat16()), lambda: drf.residual_norm(x, y, h_out=y.bfloat16()), lambda: drf.residual_norm(x, out=y),
                 lambda: drf.residual_norm(x, y, before=None, h_out=y), lambda: drf.residual_norm(x, y, lens=i[:1]), lambda: drf.residual_norm(x, y, lens=i.long()),
                 lambda: drf.residual_norm(x.transpose(1, 2), y.transpose(1, 2)),
                 lambda: drf.gated_ffn(x, w[:127], w_out), lambda: drf.gated_ffn(x, w.bfloat16(), w_out), lambda: drf.gated_ffn(x, w, w_out, b_in=v), lambda: drf.gated_ffn(x, w, w_out.t()[1:]),
                 lambda: drf.gated_ffn(x, w, w_out, out=x[:, :3]), lambda: drf.gated_ffn(x[..., :60], w, w_out),
                 lambda: drf.linear_adapters(x, w, a, b, None), lambda: drf.linear_adapters(x, w, a, b, i.long()), lambda: drf.linear_adapters(x, w, a, b[:, :5], i),
                 lambda: drf.linear_adapters(x, w, a, b, i, scales=v[:2]), lambda: drf.linear_adapters(x, w, a.bfloat16(), b, i), lambda: drf.linear_adapters(x, w, a, b, i, bias=v)):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: drf.residual_norm(x.bfloat16(), y), lambda: drf.residual_norm(x, y, out=y), lambda: drf.gated_ffn(x, w, w_out, out=x),
                 lambda: drf.gated_ffn(x, w, w_out, out=torch.zeros(1, 4, 64, device="cuda").expand(2, 4, 64)), lambda: drf.residual_norm(x, y, eps=-1.0)):
        with pytest.raises(D_.DrfError):
            call()
    with pytest.raises(KeyError):
        drf.gated_ffn(x, w, w_out, act="relu")
    empty = drf.gated_ffn(x[:, :0], w, w_out), drf.linear_adapters(x[:0], w, a, b, i[:0]), drf.residual_norm(x[:0], y[:0])[1]
    assert [tuple(e.shape) for e in empty] == [(2, 0, 64), (0, 4, 128), (0, 4, 64)]


# ---- every tile and form of the products --------------------------------------------------------------------------


@pytest.fixture
def forced(drf):
    yield drf.probe_linear_tile
    drf.probe_linear_tile(-1)


TILED = [(1, 300, 72, 80, 72), (3, 70, 64, 136, 264), (2, 260, 136, 24, 130), (5, 130, 200, 272, 300), (1, 513, 328, 136, 129), (40, 9, 448, 152, 65)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tile", range(15))
@pytest.mark.parametrize("S,N,D,F,O", TILED)
def test_gated_ffn_on_every_tile(torch, drf, forced, dtype, tile, S, N, D, F, O):
    """Tiles that rows, columns and the inner axis end inside of; slots that end inside of a tile, lengths that leave tiles empty; weights in the last step's idle columns."""
    if tile >= forced(tile):
        pytest.skip("no such tile")
    rng = np.random.default_rng(N + D)
    for layout, act in (("plain", "silu"), ("rows", "gelu"), ("tokens", "silu")):
        x, w_in, w_out, b_in, b_out = ffn_case(torch, rng, S, N, D, F, O, dtype, layout)
        want, slack = ffn(f64(x), f64(w_in), f64(w_out), f64(b_in), f64(b_out), act, dtype)
        check(drf.gated_ffn(x, w_in, w_out, b_in, b_out, act), want, dtype, slack)
        lens = [(0, N, 1, N // 2, N - 1)[j % 5] for j in range(S)]
        for j, n in enumerate(lens):
            x[j, n:] = float("nan")
        out = laid(torch, torch.full((S, N, O), 7.0, dtype=x.dtype, device="cuda"), "odd" if layout == "rows" else layout)
        drf.gated_ffn(x, w_in, w_out, b_in, b_out, act, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), out=out)
        for j, n in enumerate(lens):
            assert (out[j, n:] == 7).all()
            check(out[j, :n], want[j, :n], dtype, slack[j, :n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tile", range(15))
@pytest.mark.parametrize("R", [1, 8, 16, 24, 32, 40, 64, 72, 128, 136])
@pytest.mark.parametrize("S,N,D,_,O", TILED)
def test_linear_adapters_on_every_tile(torch, drf, forced, dtype, tile, R, S, N, D, _, O):
    """The adapter as steps of the product's loop and behind it, ranks that end inside of a step; infinite weights of one slot's adapter reach no other."""
    if tile >= forced(tile):
        pytest.skip("no such tile")
    rng = np.random.default_rng(N + D + R)
    for layout in ("plain", "tokens"):
        c = list(adapter_case(torch, rng, S, N, D, O, R, 3, dtype, layout))
        c[4] = [(1, -1, 0, 2, 2)[j % 5] for j in range(S)]
        want, slack = adapted(*[f64(v) for v in c[:4]], c[4], f64(c[5]), f64(c[6]), dtype)
        got = run_adapters(torch, drf, *c)
        check(got, want, dtype, slack)
        lens = [(N, 0, 1, N // 2, N - 1)[j % 5] for j in range(S)]
        out = torch.full_like(got, 7.0)
        y = c[0].clone()
        for j, n in enumerate(lens):
            y[j, n:] = float("nan")
        run_adapters(torch, drf, y, *c[1:], lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), out=out)
        for j, n in enumerate(lens):
            assert (out[j, n:] == 7).all()
            check(out[j, :n], want[j, :n], dtype, slack[j, :n])
        c[2], c[3] = c[2].clone(), c[3].clone()
        c[3][1, :, R - 1] = float("inf")
        others = torch.tensor([i != 1 for i in c[4]], device="cuda")
        again = run_adapters(torch, drf, *c)
        assert torch.equal(again[others], got[others]) and not torch.isfinite(again[0]).any()


def test_both_marshallings_agree(torch, drf):
    """The CPython module and ctypes make the same calls of the same arguments, and refuse the same ones."""
    x, y, rows = torch.randn(2, 5, 64, device="cuda"), torch.randn(2, 5, 64, device="cuda").bfloat16(), torch.randn(2, 5, 192, device="cuda")
    w, w_out, v, i = torch.randn(128, 64, device="cuda"), torch.randn(40, 64, device="cuda"), torch.randn(64, device="cuda"), torch.tensor([1, -1], dtype=torch.int32, device="cuda")
    a, b, lens = torch.randn(3, 6, 64, device="cuda"), torch.randn(3, 128, 6, device="cuda"), torch.tensor([5, 2], dtype=torch.int32, device="cuda")
    calls = [lambda: drf.residual_norm(x, y, gate=rows[:, 0, :64], after="rms", after_gain=v, x_scale=0.5, y_scale=2, before="layer", before_gain=v, before_bias=v, shift=rows[..., 64:128],
                                       scale=rows[..., 128:], eps=1e-3, lens=lens),
             lambda: drf.residual_norm(x), lambda: drf.residual_norm(x, y, before=None), lambda: drf.residual_norm(x, h_out=y.clone()),
             lambda: drf.gated_ffn(x, w, w_out, b_in=w[:, 0].contiguous(), b_out=v[:40], act="gelu", lens=lens), lambda: drf.gated_ffn(x[:, ::2], w, w_out),
             lambda: drf.linear_adapters(x, w, a, b, i, bias=w[:, 1].contiguous(), scales=v[:3], lens=lens), lambda: drf.linear_adapters(x, w, a[:0], b[:0], i),
             lambda: drf.gated_ffn(x[:0], w, w_out), lambda: drf.linear_adapters(x[:, :0], w, a, b, i)]
    bad = [lambda: drf.residual_norm(x, y[:1]), lambda: drf.residual_norm(x, y, out=y), lambda: drf.residual_norm(x[0]), lambda: drf.residual_norm(x, y, gate=v), lambda: drf.residual_norm(x.cpu()),
           lambda: drf.residual_norm(x, y, shift=rows[..., :63]), lambda: drf.residual_norm(x.double()), lambda: drf.residual_norm(x, y, lens=i.long()), lambda: drf.residual_norm(y, x),
           lambda: drf.residual_norm(x, before_gain=v.bfloat16()), lambda: drf.residual_norm(x, x_scale=float("inf")), lambda: drf.residual_norm(x, eps=float("nan")),
           lambda: drf.gated_ffn(x, w, w_out[:, :32]), lambda: drf.gated_ffn(y, w, w_out), lambda: drf.gated_ffn(x, w[None], w_out), lambda: drf.gated_ffn(x, w, w_out, b_in=v),
           lambda: drf.gated_ffn(x, w, w_out, out=x), lambda: drf.gated_ffn(x, w, None), lambda: drf.gated_ffn(x[..., :32], w, w_out), lambda: drf.gated_ffn(x, w.t(), w_out),
           lambda: drf.linear_adapters(x, w, a, b, None), lambda: drf.linear_adapters(x, w, a, b[:2], i), lambda: drf.linear_adapters(x, w, a[0], b, i), lambda: drf.linear_adapters(x, w, a, b, v),
           lambda: drf.linear_adapters(x, w, a, b, i, scales=v), lambda: drf.linear_adapters(x, w, a, b, i[:1]), lambda: drf.linear_adapters(x.cpu(), w, a, b, i)]
    native = drf._block_operators()
    if native is drf._BlockCtypes:
        pytest.skip("no native module for this interpreter")

    def outcome(f):
        try:
            r = f()
            return [None if t is None else t.clone() for t in (r if isinstance(r, tuple) else (r,))]
        except Exception as e:
            return e.status if isinstance(e, drf.DrfError) else AssertionError if isinstance(e, (AssertionError, AttributeError)) else type(e)
    results = []
    try:
        for form in (native, drf._BlockCtypes):
            drf._block_ops = form
            results.append([outcome(f) for f in calls + bad])
    finally:
        drf._block_ops = native
    for k, (p, q) in enumerate(zip(*results)):
        if k < len(calls):
            assert len(p) == len(q) and all(s is t if s is None or t is None else torch.equal(s, t) for s, t in zip(p, q)), k
        else:
            assert p == q and not isinstance(p, list), (k - len(calls), p, q)
