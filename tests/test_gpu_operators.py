"""The attention operators against their definitions in float64 (numpy), at the sizes, layouts and masks where they can go wrong.

Tolerances.  A rounding is off by at most half a step, 2^-8 of the value in bf16 and 2^-24 in fp32.
  rotations and norms: one rounding of the result, and fp32 arithmetic on a pair (x, y) of some 16 roundings, an angle off by 2^-22 (half a turn
      in 24 bits, pi times) and a sum of at most 128 squares (8 levels of it in a lane and across lanes): together below 2^-19 of the pair's or,
      with a norm, of the row's largest value after it.
  attention, bf16: a probability and the result are rounded to bf16, 2^-8 each, of sum p |v| / sum p and of the value; a score is a sum of d
      products in fp32, off by (d + 8) 2^-24 of scale sum |q k|, which moves every probability by that share, at most twice; 2^-18 for the rest.
  attention, fp32: the same without the first two.
Chosen blocks are whole numbers and equal the reference's."""
import numpy as np
import pytest

from paper_2603_25872_amd import drf as D_

pytestmark = pytest.mark.gpu
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


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


def tensor(torch, rng, shape, dtype, layout, scale=1.0):
    """A device tensor [slots, tokens, heads, d] in one of the memory layouts a caller may have, and its values in float64."""
    S, N, H, d = shape
    x = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(dtype_of(torch, dtype))
    if layout == "heads":
        y = torch.empty(S, H, N, d, dtype=x.dtype, device="cuda").transpose(1, 2)
    elif layout == "rows":                                                      # a column range of wider rows
        y = torch.empty(S, N, H + 2, d, dtype=x.dtype, device="cuda")[:, :, 1:1 + H]
    elif layout == "odd":                                                       # nothing is aligned to 16 bytes
        y = torch.empty(S * N * (H * (d + 3) + 1) + 1, dtype=x.dtype, device="cuda")[1:].view(S, N, H * (d + 3) + 1)[:, :, :H * (d + 3)].view(S, N, H, d + 3)[..., :d]
    else:
        y = torch.empty(S, N, H, d, dtype=x.dtype, device="cuda")
    y.copy_(x)
    return y, x.double().numpy()


def angles(cfg, S, N, positions=None):
    """[slots, tokens, pairs] and the columns of each pair, from the definition."""
    n = np.arange(N)
    out, first, second, col = [], [], [], 0
    for a in range(cfg.n_axes):
        dim = cfg.dim[a]
        if positions is None:
            below = int(np.prod([cfg.extent[b] for b in range(a + 1, cfg.n_axes)]))
            at = n // below if a == 0 else n // below % cfg.extent[a]
            pos = np.broadcast_to(cfg.origin[a] + cfg.step[a] * at, (S, N))
        else:
            pos = np.broadcast_to(positions[..., a].astype(np.float64), (S, N))
        for i in range(dim // 2):
            out.append(pos * cfg.theta ** (-2.0 * i / dim))
            pairs = cfg.layout == D_.ROPE_PAIRS
            first.append(col + (2 * i if pairs else i))
            second.append(col + (2 * i + 1 if pairs else i + dim // 2))
        col += dim
    return (np.stack(out, -1) if out else np.zeros((S, N, 0))), np.array(first, int), np.array(second, int)


def rotated(x, cfg, positions=None):
    phi, a, b = angles(cfg, x.shape[0], x.shape[1], positions)
    c, s = np.cos(phi)[:, :, None], np.sin(phi)[:, :, None]
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def normed(x, kind, gain, bias, eps):
    if kind == "layer":
        x = x - x.mean(-1, keepdims=True)
    if kind != "none":
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x * (1 if gain is None else gain) + (0 if bias is None else bias)


def check(got, want, dtype, slack):
    """|got - want| <= half a step of the result + slack, everywhere; NaN where the reference has it."""
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    bad = np.abs(got - want) > HALF[dtype] * np.abs(want) + slack
    assert not (bad & ~np.isnan(want)).any(), (int(bad.sum()), float(np.nanmax(np.abs(got - want) - HALF[dtype] * np.abs(want) - slack)))


ROTATIONS = [((72,), (1,), "pairs"), ((36, 36), (1, 9), "pairs"), ((24, 24, 24), (2, 3, 5), "halves"), ((16, 32, 16), (2, 3, 5), "halves"), ((0, 16, 8), (1, 7, 3), "halves"),
             ((6, 10, 2), (2, 3, 5), "halves"), ((2, 0, 0), (1, 1, 1), "pairs"), ((0, 0), (1, 1), "pairs")]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dims,extents,kind", ROTATIONS)
@pytest.mark.parametrize("S,N,H,layout", [(1, 1, 1, "plain"), (3, 30, 5, "rows"), (2, 37, 16, "heads"), (2, 9, 3, "odd")])
def test_rope(torch, drf, dtype, dims, extents, kind, S, N, H, layout):
    """Every section layout on vector and element accesses, one token and ragged tiles, columns that do not turn."""
    d = 72
    cfg = drf.rope_config(dims, extents, layout=kind, origin=[0.5, -3, 1000][:len(dims)], step=[0.25, 1, -2][:len(dims)])
    x, v = tensor(torch, np.random.default_rng(N + H), (S, N, H, d), dtype, layout)
    check(drf.rope(x, cfg), rotated(v, cfg), dtype, 2.0 ** -19 * np.abs(v).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,dims", [(8, (4, 2, 2)), (16, (8, 8)), (32, (32,)), (40, (8, 16, 16)), (64, (32, 32)), (80, (16, 32, 32)), (96, (32, 32, 32)), (104, (8, 48, 48)),
                                    (128, (64, 64)), (128, (128,)), (60, (20, 20, 20)), (6, (2, 4)), (1, (0,)), (127, (60, 60, 6))])
def test_rope_widths_and_tables(torch, drf, dtype, d, dims):
    """Widths that are and are not pieces of 16 bytes; positions from tables, shared and of each slot, far from zero and between numbers."""
    rng = np.random.default_rng(d)
    S, N, H = 3, 21, 4
    cfg = drf.rope_config(dims, (1,) * len(dims), theta=500.0, layout="halves" if d % 16 else "pairs")
    x, v = tensor(torch, rng, (S, N, H, d), dtype, "rows")
    for shape in ((N, len(dims)), (S, N, len(dims))):
        p = np.where(rng.random(shape) < 0.5, rng.integers(0, 2 ** 24, shape), rng.uniform(-50, 50, shape)).astype(np.float32)
        check(drf.rope(x, cfg, positions=torch.from_numpy(p).cuda()), rotated(v, cfg, p), dtype, 2.0 ** -19 * np.abs(v).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["none", "rms", "layer"])
@pytest.mark.parametrize("S,N,H,Hk,d,layout,dims,rope_layout", [
    (1, 1, 16, 16, 72, "plain", (36, 36), "pairs"), (2, 33, 6, 2, 64, "rows", (32, 16), "halves"), (3, 17, 5, 1, 128, "heads", (64, 64), "halves"),
    (2, 64, 2, 2, 32, "heads", None, None), (1, 20, 3, 3, 8, "rows", (8,), "pairs"), (2, 11, 4, 2, 72, "odd", (24, 48), "halves"), (1, 7, 2, 1, 50, "odd", None, None),
    (1, 300, 24, 8, 88, "rows", (8, 80), "pairs"), (2, 15, 7, 7, 96, "heads", (12, 12), "halves")])
def test_qk_norm_rope(torch, drf, dtype, kind, S, N, H, Hk, d, layout, dims, rope_layout):
    """Both norms and none, with and without gains and rotation, fewer key heads, a scale on the queries."""
    rng = np.random.default_rng(d + N)
    q, qv = tensor(torch, rng, (S, N, H, d), dtype, layout, 3.0)
    k, kv = tensor(torch, rng, (S, N, Hk, d), dtype, layout)
    cfg = None if dims is None else drf.rope_config(dims, (5,) * len(dims), layout=rope_layout)
    gains = [rng.uniform(0.5, 2, d).astype(np.float32) if kind != "none" and N != 33 else None for _ in range(2)]
    biases = [rng.uniform(-1, 1, d).astype(np.float32) if kind == "layer" else None for _ in range(2)]
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    qo, ko = drf.qk_norm_rope(q, k, kind, cfg, dev(gains[0]), dev(gains[1]), dev(biases[0]), dev(biases[1]), eps=1e-3, q_scale=0.3)
    for got, x, g, b, scale in ((qo, qv, gains[0], biases[0], 0.3), (ko, kv, gains[1], biases[1], 1.0)):
        y = normed(x, kind, g, b, 1e-3) * np.float64(np.float32(scale))
        check(got, y if cfg is None else rotated(y, cfg), dtype, 2.0 ** -19 * np.abs(y).max())


@pytest.mark.parametrize("layout", ["rows", "odd"])
def test_norms_in_place_and_rows_behind_a_length(torch, drf, layout):
    """In place; lengths of zero, one, all and more; what lies behind them, not numbers included, is neither read into a result nor written."""
    rng = np.random.default_rng(1)
    S, N, H, d = 5, 19, 3, 40
    lens = np.array([0, 1, 19, 25, -4], np.int32)
    cfg = drf.rope_config((20, 20), (1, 4), layout="halves")
    q, qv = tensor(torch, rng, (S, N, H, d), "bf16", layout)
    k, kv = tensor(torch, rng, (S, N, H, d), "bf16", layout)
    inside = (np.arange(N)[None] < lens[:, None])[:, :, None, None]
    mask = torch.from_numpy(np.broadcast_to(inside, (S, N, H, d)).copy()).cuda()
    q[~mask] = float("nan")
    got = drf.qk_norm_rope(q, k, "rms", cfg, lens=torch.from_numpy(lens).cuda(), q_out=q, k_out=k)
    assert got[0] is q and got[1] is k
    for t, v in ((q, qv), (k, kv)):
        y = rotated(normed(v, "rms", None, None, 1e-6), cfg)
        check(torch.where(mask, t, torch.zeros_like(t)), np.where(inside, y, 0.0), "bf16", 2.0 ** -19 * np.abs(y).max())
    assert torch.isnan(q[~mask]).all() and torch.equal(k[~mask].cpu(), torch.from_numpy(kv)[~mask.cpu()].to(torch.bfloat16))
    x = torch.randn(S, N, H, d, device="cuda")
    out = torch.full_like(x, 7.0)
    drf.rope(x, cfg, lens=torch.from_numpy(lens).cuda(), out=out)
    assert (out[~mask] == 7.0).all() and not (out[mask] == 7.0).any()


def test_turning_back_gives_the_input(torch, drf):
    """The rotation with origins and steps negated is its inverse, and its transpose: what a gradient is turned by."""
    x = torch.randn(2, 100, 3, 64, device="cuda")
    there, back = drf.rope_config((20, 44), (1, 10), origin=(3, 4)), drf.rope_config((20, 44), (1, 10), origin=(-3, -4), step=(-1, -1))
    assert (drf.rope(drf.rope(x, there), back) - x).abs().max() <= 2.0 ** -18 * x.abs().max()
    g = torch.randn_like(x)
    left, right = (drf.rope(x, there).double() * g).sum(), (x.double() * drf.rope(g, back)).sum()
    assert abs(float(left - right)) <= 2.0 ** -18 * float((x.abs() * g.abs()).sum())


# ---- which blocks -------------------------------------------------------------------------------------


def chosen(q, k, q_block, kv_block, topk, q_lens=None, kv_lens=None):
    """Booleans [slots, heads, query blocks, key blocks] from the definition."""
    S, N, H, d = q.shape
    M, group = k.shape[1], H // k.shape[2]
    nq, nk = -(-N // q_block), -(-M // kv_block)
    out = np.zeros((S, H, nq, nk), bool)
    for s in range(S):
        n = N if q_lens is None else min(max(int(q_lens[s]), 0), N)
        m = M if kv_lens is None else min(max(int(kv_lens[s]), 0), M)
        for h in range(H):
            live = -(-m // kv_block)
            means = [k[s, j * kv_block:min((j + 1) * kv_block, m), h // group].mean(0) for j in range(live)]
            for i in range(-(-n // q_block)):
                qm = q[s, i * q_block:min((i + 1) * q_block, n), h].mean(0)
                score = [(-np.inf, 1) if np.isnan(qm @ km) else (float(qm @ km), 0) for km in means]
                order = sorted(range(live), key=lambda j: (score[j][1], -score[j][0], j))
                out[s, h, i, order[:topk]] = True
    return out


def bits(torch, words, nk):
    w = words.cpu().numpy().view(np.uint32)
    b = (w[..., None] >> np.arange(32, dtype=np.uint32)) & 1
    b = b.reshape(*w.shape[:-1], -1).astype(bool)
    assert not b[..., nk:].any()
    return b[..., :nk]


def pack(torch, mask):
    words = -(-mask.shape[-1] // 32)
    b = np.zeros((*mask.shape[:-1], words * 32), np.uint32)
    b[..., :mask.shape[-1]] = mask
    w = (b.reshape(*mask.shape[:-1], words, 32) << np.arange(32, dtype=np.uint32)).sum(-1, dtype=np.uint32)
    return torch.from_numpy(w.view(np.int32).copy()).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,N,M,H,Hk,d,q_block,kv_block,topk,layout", [
    (1, 1, 1, 1, 1, 8, 32, 32, 1, "plain"), (2, 300, 300, 4, 2, 72, 64, 64, 2, "rows"), (1, 1, 2000, 3, 3, 64, 128, 32, 7, "heads"), (2, 129, 700, 5, 1, 40, 128, 128, 3, "rows"),
    (1, 530, 2080, 2, 2, 128, 32, 32, 33, "heads"), (1, 65, 4097, 1, 1, 16, 64, 32, 128, "plain"), (2, 100, 260, 2, 1, 72, 32, 64, 2, "odd"), (1, 70, 9000, 2, 1, 8, 64, 32, 40, "heads"),
    (1, 33, 32768, 1, 1, 8, 32, 32, 1023, "plain"), (1, 96, 200, 17, 17, 24, 32, 32, 9, "rows")])
def test_block_select(torch, drf, dtype, S, N, M, H, Hk, d, q_block, kv_block, topk, layout):
    rng = np.random.default_rng(N + M)
    q, qv = tensor(torch, rng, (S, N, H, d), dtype, layout)
    k, kv = tensor(torch, rng, (S, M, Hk, d), dtype, layout)
    got = bits(torch, drf.block_select(q, k, q_block, kv_block, topk), -(-M // kv_block))
    assert np.array_equal(got, chosen(qv, kv, q_block, kv_block, topk))


def test_block_select_odd_fp32_width(torch, drf):
    rng = np.random.default_rng(4)
    (q, qv), (k, kv) = (tensor(torch, rng, (2, n, 3, 37), "f32", "plain") for n in (70, 210))
    assert np.array_equal(bits(torch, drf.block_select(q, k, 32, 32, 3), 7), chosen(qv, kv, 32, 32, 3))


def test_block_select_lengths(torch, drf):
    """No query, no key, part of a block, more than there is; rows behind a length hold what is not a number."""
    rng = np.random.default_rng(5)
    S, N, H, d = 6, 200, 2, 32
    q_lens, kv_lens = np.array([0, 1, 33, 200, 999, 64], np.int32), np.array([50, 0, 1, 65, 200, -1], np.int32)
    (q, qv), (k, kv) = (tensor(torch, rng, (S, N, H, d), "bf16", "rows") for _ in range(2))
    for t, lens in ((q, q_lens), (k, kv_lens)):
        t[torch.from_numpy(np.arange(N)[None] >= lens[:, None]).cuda()] = float("nan")
    got = bits(torch, drf.block_select(q, k, 32, 64, 2, q_lens=torch.from_numpy(q_lens).cuda(), kv_lens=torch.from_numpy(kv_lens).cuda()), 4)
    assert np.array_equal(got, chosen(qv, kv, 32, 64, 2, q_lens, kv_lens))
    assert not got[0].any() and not got[1].any() and got[4].sum(-1).min() == 2


def test_block_select_ties_and_numbers_that_are_none(torch, drf):
    """Equal scores go to the lower block, zeros of both signs are equal, a block with an infinity or a NaN keeps its place in the order."""
    q = torch.zeros(1, 32, 1, 8, device="cuda")
    k = torch.randn(1, 32 * 40, 1, 8, device="cuda")
    assert np.array_equal(bits(torch, drf.block_select(q, k, 32, 32, 7), 40)[0, 0, 0], np.arange(40) < 7)         # all scores are +-0
    q += 1.0
    k = torch.full_like(k, 0.25)
    assert np.array_equal(bits(torch, drf.block_select(q, k, 32, 32, 33), 40)[0, 0, 0], np.arange(40) < 33)
    kb = k.view(40, 32, 8)
    kb[[3, 35]] = 0.5                                                                                             # two above, the rest equal
    kb[7, 5, 2], kb[9, 0, 0], kb[11, 1, 1] = float("nan"), float("inf"), float("-inf")
    got = bits(torch, drf.block_select(q, k, 32, 32, 5), 40)[0, 0, 0]
    assert np.flatnonzero(got).tolist() == [0, 1, 3, 9, 35]
    got = bits(torch, drf.block_select(q, k, 32, 32, 39), 40)[0, 0, 0]
    assert np.flatnonzero(~got).tolist() == [7]                                                                   # behind -infinity
    assert bits(torch, drf.block_select(q, k, 32, 32, 1000), 40).all()


def test_block_select_sums_hide_nothing(torch, drf):
    """Blocks whose means differ in the last bits only: what a sum in 32 bits would confuse."""
    k = torch.ones(1, 64 * 8, 1, 8, device="cuda").view(8, 64, 8)
    for j in range(8):
        k[j, :, 0] = 4096.0
        k[j, 63, 0] += (j * 5 % 8) * 2.0 ** -11                                                                   # 2^-29 of the sum a step
    q = torch.zeros(1, 32, 1, 8, device="cuda")
    q[..., 0] = 3.0
    got = bits(torch, drf.block_select(q, k.view(1, 512, 1, 8), 32, 64, 3), 8)[0, 0, 0]
    assert np.flatnonzero(got).tolist() == sorted(np.argsort([-(j * 5 % 8) for j in range(8)])[:3].tolist())


# ---- attention over them --------------------------------------------------------------------------------


def attended(q, k, v, mask, q_block, kv_block, scale, q_lens=None, kv_lens=None):
    """(result, sum p |v| / sum p, largest scale sum |q k| of a query's keys), rows outside a length 0."""
    S, N, H, d = q.shape
    M, group = k.shape[1], H // k.shape[2]
    out, mag, size = np.zeros_like(q), np.zeros_like(q), np.zeros((S, N, H, 1))
    for s in range(S):
        n = N if q_lens is None else min(max(int(q_lens[s]), 0), N)
        m = M if kv_lens is None else min(max(int(kv_lens[s]), 0), M)
        for h in range(H):
            for i in range(-(-n // q_block)):
                rows = slice(i * q_block, min((i + 1) * q_block, n))
                keys = np.flatnonzero(np.repeat(mask[s, h, i], kv_block)[:m]) if m else np.zeros(0, int)
                if keys.size == 0:
                    continue
                qq, kk, vv = q[s, rows, h], k[s, keys, h // group], v[s, keys, h // group]
                sc = scale * (qq @ kk.T)
                top = sc.max(1, keepdims=True)
                p = np.exp(sc - np.where(np.isinf(top) & (top < 0), 0, top))
                tot = p.sum(1, keepdims=True)
                with np.errstate(invalid="ignore"):
                    out[s, rows, h] = np.where(tot == 0, 0, (p @ vv) / np.where(tot == 0, 1, tot))
                    mag[s, rows, h] = np.where(tot == 0, 0, (p @ np.abs(vv)) / np.where(tot == 0, 1, tot))
                fine = np.where(np.isfinite(kk), np.abs(kk), 0)
                size[s, rows, h] = (scale * (np.abs(qq) @ fine.T)).max(1, keepdims=True)
    return out, mag, size


def slack_of(dtype, d, mag, size):
    return mag * ((2.0 ** -8 if dtype == "bf16" else 0) + 2 * (d + 8) * 2.0 ** -24 * size + 2.0 ** -18)


def attend(torch, drf, dtype, S, N, M, H, Hk, d, q_block, kv_block, mask, layout="rows", scale=None, scales=(1, 1, 1), q_lens=None, kv_lens=None, seed=0, split=False):
    rng = np.random.default_rng(seed + N + M + d)
    (q, qv), (k, kv), (v, vv) = (tensor(torch, rng, (S, n, h, d), dtype, layout, f) for n, h, f in zip((N, M, M), (H, Hk, Hk), scales))
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    got = drf.block_attention(q, k, v, pack(torch, mask), q_block, kv_block, scale, dev(q_lens), dev(kv_lens), split=split)
    want, mag, size = attended(qv, kv, vv, mask, q_block, kv_block, d ** -0.5 if scale is None else scale, q_lens, kv_lens)
    check(got, want, dtype, slack_of(dtype, d, mag, size))


def random_mask(rng, S, H, N, M, q_block, kv_block, share):
    return rng.random((S, H, -(-N // q_block), -(-M // kv_block))) < share


@pytest.mark.parametrize("dtype,d", [("bf16", d) for d in range(8, 129, 8)] + [("f32", d) for d in (1, 7, 16, 30, 32, 50, 64, 72, 100, 128)])
@pytest.mark.parametrize("N,M,q_block,kv_block", [(1, 33, 32, 32), (100, 257, 32, 64), (200, 390, 64, 32), (300, 300, 128, 128), (257, 1100, 64, 64)])
def test_block_attention_widths(torch, drf, dtype, d, N, M, q_block, kv_block):
    """Every width; a key block, a query block and a step that the tokens end inside of; some rows of the mask empty."""
    mask = random_mask(np.random.default_rng(d + N), 2, 4, N, M, q_block, kv_block, 0.4)
    attend(torch, drf, dtype, 2, N, M, 4, 2, d, q_block, kv_block, mask)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_block", [32, 64, 128])
@pytest.mark.parametrize("kv_block", [32, 64, 128])
@pytest.mark.parametrize("N", [1, 31, 64, 65, 400])
def test_block_attention_blocks(torch, drf, dtype, q_block, kv_block, N):
    M = 1000
    mask = random_mask(np.random.default_rng(N), 1, 3, N, M, q_block, kv_block, 0.3)
    attend(torch, drf, dtype, 1, N, M, 3, 1, 64, q_block, kv_block, mask, layout="heads", scale=0.3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 72])
@pytest.mark.parametrize("kind", ["none", "first", "last", "one", "all"])
def test_block_attention_masks(torch, drf, dtype, d, kind):
    """Masks that leave nothing, a single block at either end, everything (more than 32 blocks: more than one word)."""
    N, M, qb, kb = 130, 40 * 32 - 5, 64, 32
    mask = np.zeros((1, 2, 3, 40), bool)
    if kind == "first":
        mask[..., 0] = True
    elif kind == "last":
        mask[..., 39] = True
    elif kind == "one":
        mask[:, 0, 1, 33] = True
    elif kind == "all":
        mask[...] = True
    attend(torch, drf, dtype, 1, N, M, 2, 2, d, qb, kb, mask)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 72, 128])
def test_block_attention_scores_that_grow(torch, drf, dtype, d):
    """Scores of tens of units that grow along the keys: the reference of the softmax moves again and again."""
    rng = np.random.default_rng(d)
    N, M = 96, 640
    (q, qv), (k, kv), (v, vv) = (tensor(torch, rng, (1, n, 2, d), dtype, "plain") for n in (N, M, M))
    grow = torch.linspace(0.2, 16, M, device="cuda").view(1, M, 1, 1)
    q, k = (q * 2).to(q.dtype), (k * grow).to(k.dtype)
    mask = random_mask(rng, 1, 2, N, M, 32, 32, 0.7)
    want, mag, size = attended(q.double().cpu().numpy(), k.double().cpu().numpy(), vv, mask, 32, 32, d ** -0.5)
    check(drf.block_attention(q, k, v, pack(torch, mask), 32, 32), want, dtype, slack_of(dtype, d, mag, size))
    k = k.flip(1)                                                               # and the largest first
    want, mag, size = attended(q.double().cpu().numpy(), k.double().cpu().numpy(), vv, mask, 32, 32, d ** -0.5)
    check(drf.block_attention(q, k, v, pack(torch, mask), 32, 32), want, dtype, slack_of(dtype, d, mag, size))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [40, 64, 72])
def test_block_attention_lengths_and_masked_places(torch, drf, dtype, d):
    """Lengths of zero, one and part of a step; what is not a number in blocks that are not chosen and behind the lengths stays out, and rows of
    the output behind a query length stay as they were."""
    rng = np.random.default_rng(d)
    S, N, H, qb, kb = 6, 170, 2, 64, 32
    q_lens, kv_lens = np.array([0, 1, 65, 170, 500, 128], np.int32), np.array([170, 33, 0, 169, 1, -7], np.int32)
    mask = random_mask(rng, S, H, N, N, qb, kb, 0.5)
    mask[:, 1] = mask[:, 0]                                                     # both heads skip the same blocks
    (q, qv), (k, kv), (v, vv) = (tensor(torch, rng, (S, N, H, d), dtype, "rows") for _ in range(3))
    used = np.repeat(mask.any((1, 2)), kb, axis=1)[:, :N] & (np.arange(N)[None] < kv_lens[:, None])
    for t in (k, v):
        t[torch.from_numpy(~used).cuda()] = float("nan")
    q[torch.from_numpy(np.arange(N)[None] >= q_lens[:, None]).cuda()] = float("inf")
    out = torch.full((S, N, H, d), 7.0, dtype=q.dtype, device="cuda")
    drf.block_attention(q, k, v, pack(torch, mask), qb, kb, None, torch.from_numpy(q_lens).cuda(), torch.from_numpy(kv_lens).cuda(), out=out)
    want, mag, size = attended(qv, np.where(used[:, :, None, None], kv, 0), np.where(used[:, :, None, None], vv, 0), mask, qb, kb, d ** -0.5, q_lens, kv_lens)
    inside = np.broadcast_to((np.arange(N)[None] < q_lens[:, None])[:, :, None, None], want.shape)
    check(out, np.where(inside, want, 7.0), dtype, slack_of(dtype, d, mag, size))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_block_attention_scores_of_minus_infinity(torch, drf, dtype):
    """Keys that score -infinity are keys with no weight, first, among others and alone (no weight at all: zeros)."""
    N, M, d = 40, 160, 64
    rng = np.random.default_rng(3)
    (q, qv), (k, kv), (v, vv) = (tensor(torch, rng, (1, n, 1, d), dtype, "plain") for n in (N, M, M))
    q, qv = q.abs(), np.abs(qv)
    q[..., 0] = 1.0
    qv[..., 0] = 1.0
    kv[:, :64, :, 0] = kv[:, 100:, :, 0] = -np.inf
    k.copy_(torch.from_numpy(kv))
    for cols in ([0, 1, 2, 3, 4], [0, 1], [4, 2], [4]):
        mask = np.zeros((1, 1, 2, 5), bool)
        mask[..., cols] = True
        want, mag, size = attended(qv, kv, vv, mask, 32, 32, d ** -0.5)
        check(drf.block_attention(q, k, v, pack(torch, mask), 32, 32), want, dtype, slack_of(dtype, d, mag, size))


def many(torch, drf, q, k, v, mask, qv, kv, vv, q_block, kv_block, tiles, q_lens=None, kv_lens=None, out=None, scale=None):
    """Attention on as many copies of the slots as give `tiles` 32-query tiles (how many there are chooses how waves share them): every copy's
    result is the first one's, which has the float64 result."""
    S, N, H, d = q.shape
    c = -(-tiles // (-(-N // 32) * H * S))
    more = lambda t: None if t is None else t.repeat((c,) + (1,) * (t.dim() - 1))  # noqa: E731
    dev = lambda a: None if a is None else more(torch.from_numpy(a).cuda())  # noqa: E731
    got = drf.block_attention(more(q), more(k), more(v), more(pack(torch, mask)), q_block, kv_block, scale, dev(q_lens), dev(kv_lens), out=more(out))
    want, mag, size = attended(qv, kv, vv, mask, q_block, kv_block, d ** -0.5 if scale is None else scale, q_lens, kv_lens)
    if out is not None:
        inside = np.broadcast_to((np.arange(N)[None] < (np.full(S, N) if q_lens is None else q_lens)[:, None])[:, :, None, None], want.shape)
        want = np.where(inside, want, out.double().cpu().numpy())
    check(got[:S], want, "bf16", slack_of("bf16", d, mag, size))
    got = got.view(torch.int16).view(c, S, N, H, d)
    assert torch.equal(got, got[:1].expand_as(got))


# Tiles where a wave takes 32 queries of its own, and 64.
TILES = [600, 1100]


@pytest.mark.parametrize("tiles", TILES)
@pytest.mark.parametrize("d", range(8, 129, 8))
@pytest.mark.parametrize("N,M,q_block,kv_block", [(1, 33, 32, 32), (97, 257, 128, 64), (200, 390, 64, 32), (65, 64, 64, 64), (130, 700, 128, 128)])
def test_block_attention_of_many_tiles(torch, drf, tiles, d, N, M, q_block, kv_block):
    rng = np.random.default_rng(d + N)
    (q, qv), (k, kv), (v, vv) = (tensor(torch, rng, (2, n, h, d), "bf16", "rows") for n, h in ((N, 4), (M, 2), (M, 2)))
    many(torch, drf, q, k, v, random_mask(rng, 2, 4, N, M, q_block, kv_block, 0.5), qv, kv, vv, q_block, kv_block, tiles)


@pytest.mark.parametrize("tiles", TILES)
@pytest.mark.parametrize("d", [24, 64, 72, 128])
@pytest.mark.parametrize("steepest", [1.0, 4.0, 16.0])
@pytest.mark.parametrize("qb", [64, 128])
def test_block_attention_of_many_tiles_scores_that_grow(torch, drf, tiles, d, steepest, qb):
    """The first step's scores are small, later ones larger: by what sums in fp32 hold beside them, and by far more."""
    rng = np.random.default_rng(d)
    N, M = 96, 640
    (q, _), (k, _), (v, vv) = (tensor(torch, rng, (1, n, 2, d), "bf16", "plain") for n in (N, M, M))
    q, k = (q * 2).to(q.dtype), (k * torch.linspace(0.2, steepest, M, device="cuda").view(1, M, 1, 1)).to(k.dtype)
    for turn in (k, k.flip(1)):
        many(torch, drf, q, turn, v, random_mask(rng, 1, 2, N, M, qb, 32, 0.7), q.double().cpu().numpy(), turn.double().cpu().numpy(), vv, qb, 32, tiles)


@pytest.mark.parametrize("tiles", [1] + TILES)
@pytest.mark.parametrize("d", [40, 64, 72, 104])
@pytest.mark.parametrize("qb", [64, 128])
def test_block_attention_of_many_tiles_lengths_and_masked_places(torch, drf, tiles, d, qb):
    rng = np.random.default_rng(d)
    S, N, H, kb = 6, 170, 2, 32
    q_lens, kv_lens = np.array([0, 1, 65, 170, 500, 128], np.int32), np.array([170, 33, 0, 169, 1, -7], np.int32)
    mask = random_mask(rng, S, H, N, N, qb, kb, 0.5)
    mask[:, 1] = mask[:, 0]
    (q, qv), (k, kv), (v, vv) = (tensor(torch, rng, (S, N, H, d), "bf16", "rows") for _ in range(3))
    used = np.repeat(mask.any((1, 2)), kb, axis=1)[:, :N] & (np.arange(N)[None] < kv_lens[:, None])
    for t in (k, v):
        t[torch.from_numpy(~used).cuda()] = float("nan")
    q[torch.from_numpy(np.arange(N)[None] >= q_lens[:, None]).cuda()] = float("inf")
    out = torch.full((S, N, H, d), 7.0, dtype=q.dtype, device="cuda")
    kv, vv = (np.where(used[:, :, None, None], x, 0) for x in (kv, vv))
    many(torch, drf, q, k, v, mask, qv, kv, vv, qb, kb, tiles, q_lens, kv_lens, out)


@pytest.mark.parametrize("tiles", [1] + TILES)
@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("qb", [64, 128])
def test_block_attention_behind_a_step_of_no_weight(torch, drf, tiles, d, qb):
    """A list's first keys score -infinity, the others so low that their exponentials alone would vanish."""
    rng = np.random.default_rng(d)
    N, M = 96, 160
    (q, qv), (k, kv), (v, vv) = (tensor(torch, rng, (1, n, 2, d), "bf16", "plain") for n in (N, M, M))
    q[..., 0] = 1.0
    qv[..., 0] = 1.0
    q[..., 1:], qv[..., 1:] = q[..., 1:] / 4, qv[..., 1:] / 4                  # (exact)
    kv[:, :64, :, 0], kv[:, 64:, :, 0] = -np.inf, -8192.0
    k.copy_(torch.from_numpy(kv))
    mask = np.ones((1, 2, -(-N // qb), 5), bool)
    mask[0, 1, -1] = [1, 0, 0, 0, 1]
    many(torch, drf, q, k, v, mask, qv, kv, vv, qb, 32, tiles)


@pytest.mark.parametrize("S,N,M", [(0, 5, 5), (2, 0, 40), (2, 40, 0)])
def test_operators_of_nothing(torch, drf, S, N, M):
    q, k = (torch.randn(S, n, 2, 64, device="cuda").bfloat16() for n in (N, M))
    cfg = drf.rope_config((64,), (1,))
    assert drf.rope(q, cfg).shape == q.shape
    assert drf.qk_norm_rope(q, q, "rms", cfg)[0].shape == q.shape
    words = drf.block_select(q, k, 32, 32, 2)
    assert words.shape == (S, 2, -(-N // 32), -(-M // 32 // 32))
    assert not drf.block_attention(q, k, k, words, 32, 32).any()


@pytest.mark.parametrize("d", [32, 48, 64, 72, 96, 128])
@pytest.mark.parametrize("layout", ["odd", "heads"])
def test_block_attention_fp32_layouts(torch, drf, d, layout):
    """Rows and heads that are not aligned to 16 bytes, and heads that lie outside of the tokens."""
    attend(torch, drf, "f32", 2, 70, 200, 4, 2, d, 32, 32, random_mask(np.random.default_rng(d), 2, 4, 70, 200, 32, 32, 0.5), layout=layout)


@pytest.mark.parametrize("d", [8, 40, 64, 72, 96, 128])
@pytest.mark.parametrize("N,M,H,kv_block,share", [(1, 8192, 2, 64, 0.5), (33, 8200, 3, 32, 0.02), (1, 9000, 16, 128, 1.0), (5, 20000, 1, 32, 0.7), (64, 8255, 2, 128, 0.3), (1, 8192, 64, 64, 0.1)])
def test_block_attention_of_few_queries_over_many_keys(torch, drf, d, N, M, H, kv_block, share):
    """Several workgroups to a head: lists of every length, parts with no step, lengths that leave most of the keys or all of them out."""
    rng = np.random.default_rng(N + d)
    kv_heads = 1 if H % 2 else H // 2
    mask = random_mask(rng, 1, H, N, M, 32, kv_block, share)
    mask[:, 0, 0] = 0
    attend(torch, drf, "bf16", 1, N, M, H, kv_heads, d, 32, kv_block, mask, layout="rows", split=True)
    mask[:, 0, 0, -1] = 1                                                       # one block, which the keys end inside of
    for length in (M - 1, 700, 1, 0):
        attend(torch, drf, "bf16", 1, N, M, H, kv_heads, d, 32, kv_block, mask, layout="heads", kv_lens=np.array([length], np.int32), split=True)


def test_block_attention_parts_in_a_replayed_graph_and_beside_the_unsplit_call(torch, drf):
    rng = np.random.default_rng(4)
    (q, qv), (k, kv), (v, vv) = (tensor(torch, rng, (2, n, 2, 64), "bf16", "plain") for n in (3, 8192, 8192))
    mask = random_mask(rng, 2, 2, 3, 8192, 32, 64, 0.4)
    words, lens, out = pack(torch, mask), torch.tensor([2, 3], dtype=torch.int32, device="cuda"), torch.full((2, 3, 2, 64), 7.0, dtype=q.dtype, device="cuda")
    run = lambda: drf.block_attention(q, k, v, words, 32, 64, None, lens, out=out, split=True)  # noqa: E731
    want, mag, size = attended(qv, kv, vv, mask, 32, 64, 0.125, np.array([2, 3]))
    want[0, 2] = 7.0
    for t in (torch.cuda.current_stream(), torch.cuda.Stream()):
        t.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(t):
            run()
        torch.cuda.current_stream().wait_stream(t)
        check(out, want, "bf16", slack_of("bf16", 64, mag, size))
    eager, g = out.clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for _ in range(3):
        out[0, :2] = out[1] = 0.0
        g.replay()
        assert torch.equal(out, eager)
        run()
        assert torch.equal(out, eager)
    whole = torch.full_like(out, 7.0)
    hs = [drf._heads(t) for t in (q, k, v, whole)]
    shape = drf.AttnShape(drf.BF16, 2, 3, 8192, 2, 2, 64, lens.data_ptr(), None)
    assert drf.lib().drf_block_attention(drf.C.byref(shape), 32, 64, 0.125, words.data_ptr(), *[drf.C.byref(h) for h in hs], drf._current(q)) == 0
    check(whole, want, "bf16", slack_of("bf16", 64, mag, size))


def test_block_attention_ignores_bits_behind_the_last_block(torch, drf):
    rng = np.random.default_rng(8)
    (q, _), (k, _), (v, _) = (tensor(torch, rng, (1, 70, 2, 64), "bf16", "plain") for _ in range(3))
    mask = random_mask(rng, 1, 2, 70, 70, 32, 32, 0.6)
    w = pack(torch, mask)
    want = drf.block_attention(q, k, v, w, 32, 32)
    assert torch.equal(drf.block_attention(q, k, v, w | ~7, 32, 32), want)


def test_offsets_beyond_32_bits(torch, drf):
    """Slots and heads more than 2^31 elements apart: views of one allocation of 8.6 GB, of which little is touched."""
    S, N, H, d = 2, 70, 2, 64
    big = torch.empty(S, H, 2 ** 30, dtype=torch.bfloat16, device="cuda")
    views = [big[:, :, i * 10 ** 6 + 8:][:, :, :N * d].view(S, H, N, d).transpose(1, 2) for i in range(4)]
    rng = np.random.default_rng(2)
    vals = [tensor(torch, rng, (S, N, H, d), "bf16", "plain") for _ in range(3)]
    for view, (t, _) in zip(views, vals):
        view.copy_(t)
    q, k, v = views[:3]
    cfg = drf.rope_config((32, 32), (1, 9))
    check(drf.rope(q, cfg, out=views[3]), rotated(vals[0][1], cfg), "bf16", 2.0 ** -19 * np.abs(vals[0][1]).max())
    words = drf.block_select(q, k, 32, 32, 2)
    mask = bits(torch, words, 3)
    assert np.array_equal(mask, chosen(vals[0][1], vals[1][1], 32, 32, 2))
    want, mag, size = attended(vals[0][1], vals[1][1], vals[2][1], mask, 32, 32, d ** -0.5)
    check(drf.block_attention(q, k, v, words, 32, 32, out=views[3]), want, "bf16", slack_of("bf16", d, mag, size))


# ---- together ---------------------------------------------------------------------------------------------


def chain(drf, qkv, cfg, gains, q_block, kv_block, topk, lens=None):
    """The operators as an attention layer runs them: q and k of a qkv Linear's rows in place, the choice, the attention."""
    q, k, v = qkv.unbind(2)
    drf.qk_norm_rope(q, k, "rms", cfg, gains, gains, lens=lens, q_out=q, k_out=k)
    words = drf.block_select(q, k, q_block, kv_block, topk, q_lens=lens, kv_lens=lens)
    return words, drf.block_attention(q, k, v, words, q_block, kv_block, q_lens=lens, kv_lens=lens)


@pytest.mark.parametrize("dtype,S,N,H,d", [("bf16", 3, 420, 4, 72), ("f32", 2, 256, 2, 32), ("bf16", 1, 1, 3, 64)])
def test_the_operators_together(torch, drf, dtype, S, N, H, d):
    rng = np.random.default_rng(N)
    x = torch.from_numpy(rng.standard_normal((S, N, 3, H, d)).astype(np.float32)).to(dtype_of(torch, dtype)).cuda()
    gains = torch.linspace(0.5, 1.5, d, device="cuda")
    cfg = drf.rope_config((d // 2 // 4 * 4, d // 4 // 4 * 4), (1, 20))
    lens = np.minimum(N, np.array([N, N // 2 + 1, 0][:S])).astype(np.int32)
    work = x.clone()
    words, got = chain(drf, work, cfg, gains, 64, 32, 4, torch.from_numpy(lens).cuda())
    q, k, v = (t.squeeze(2) for t in np.split(x.double().cpu().numpy(), 3, axis=2))
    inside = (np.arange(N)[None] < lens[:, None])[:, :, None, None]
    for i, t in enumerate((q, k)):
        y = np.where(inside, rotated(normed(t, "rms", gains.double().cpu().numpy(), None, 1e-6), cfg), t)
        check(work[:, :, i], y, dtype, 2.0 ** -19 * np.abs(y).max())
    qn, kn = (work[:, :, i].double().cpu().numpy() for i in range(2))           # the choice and the attention go by the rounded q and k
    mask = chosen(qn, kn, 64, 32, 4, lens, lens)
    assert np.array_equal(bits(torch, words, mask.shape[-1]), mask)
    want, mag, size = attended(qn, kn, v, mask, 64, 32, d ** -0.5, lens, lens)
    check(got, want, dtype, slack_of(dtype, d, mag, size))


def test_captured_and_replayed_between_eager_calls(torch, drf):
    """Two graphs of the chain and eager calls in between, replayed several times: every result is the eager one, bit for bit."""
    torch.manual_seed(0)
    cfg, gains = drf.rope_config((36, 36), (1, 16)), torch.ones(72, device="cuda")
    inputs = [torch.randn(2, 256, 3, 4, 72, device="cuda").bfloat16() for _ in range(3)]
    want = [[t.clone() for t in chain(drf, x.clone(), cfg, gains, 64, 64, 2)] for x in inputs]
    graphs = []
    for _ in range(2):
        held = inputs[0].clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = chain(drf, held, cfg, gains, 64, 64, 2)
        graphs.append((g, held, out))
    for it in range(4):
        for n, (g, held, out) in enumerate(graphs):
            held.copy_(inputs[(it + n) % 3])
            g.replay()
            eager = chain(drf, inputs[it % 3].clone(), cfg, gains, 64, 64, 2)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want[(it + n) % 3])), (it, n)
            assert all(torch.equal(a, b) for a, b in zip(eager, want[it % 3])), it


def test_two_streams_at_once(torch, drf):
    """Calls on two streams share nothing: each gives what it gives alone."""
    torch.manual_seed(1)
    cfg, gains = drf.rope_config((32, 32), (1, 32)), torch.ones(64, device="cuda")
    xs = [torch.randn(2, 1024, 3, 6, 64, device="cuda").bfloat16() for _ in range(2)]
    want = [[t.clone() for t in chain(drf, x.clone(), cfg, gains, 64, 64, 4)] for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for x, st in zip(xs, streams):
            with torch.cuda.stream(st):
                got.append(chain(drf, x.clone(), cfg, gains, 64, 64, 4))
    torch.cuda.synchronize()
    for n, g in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, want[n % 2])), n


# ---- the binding -------------------------------------------------------------------------------------------


def test_both_marshallings_give_the_same(torch, drf, monkeypatch):
    """The calls through the CPython module and through ctypes: results bit for bit, and the same tensors refused before anything is launched."""
    torch.manual_seed(2)
    x = torch.randn(2, 70, 3, 4, 64, device="cuda").bfloat16()
    cfg, gains, lens = drf.rope_config((32, 32), (1, 9)), torch.rand(64, device="cuda"), torch.tensor([70, 31], dtype=torch.int32, device="cuda")
    table = torch.rand(2, 70, 2, device="cuda")
    q, k, v = x.unbind(2)
    f = q.float()
    words = drf.block_select(q, k, 32, 32, 2)
    far, some = torch.randn(2, 8192, 4, 64, device="cuda").bfloat16(), torch.full((2, 4, 1, 8), 0x1234567, dtype=torch.int32, device="cuda")
    forms = (drf._operators(), drf._OperatorsCtypes)
    assert forms[0] is not forms[1]                                             # built beside the library here
    got = []
    for form in forms:
        monkeypatch.setattr(drf, "_ops", form)
        out = [drf.rope(q, cfg), drf.rope(f, cfg, positions=table, lens=lens), *chain(drf, x.clone(), cfg, gains, 32, 64, 1, lens),
               *drf.qk_norm_rope(q, k[:, :, :2], "layer", None, gains, gains, gains, gains, q_scale=2.0), drf.block_attention(q, k, v, words, 32, 32, scale=0.5),
               drf.block_attention(q[:, :2], far, far, some, 32, 32, split=True), drf.block_attention(q, k, v, words, 32, 32, split=True)]
        bad = []
        for call in (lambda: drf.rope(q, cfg, out=f), lambda: drf.rope(q, cfg, out=k[:, :69]), lambda: drf.rope(q[0], cfg), lambda: drf.rope(q.half(), cfg),
                     lambda: drf.rope(q.transpose(2, 3), cfg), lambda: drf.rope(q.cpu(), cfg), lambda: drf.rope(q, cfg, lens=lens.long()), lambda: drf.rope(q, cfg, lens=lens[:1]),
                     lambda: drf.rope(q, cfg, lens=lens.cpu()), lambda: drf.rope(q, cfg, positions=table[:, :, :1]), lambda: drf.rope(q, cfg, positions=table[0, 0]),
                     lambda: drf.qk_norm_rope(q, k, "rms", None, positions=table), lambda: drf.qk_norm_rope(q, k[:, 1:], "rms"), lambda: drf.qk_norm_rope(q, k, "rms", q_gain=gains[1:]),
                     lambda: drf.qk_norm_rope(q, k, "none", q_gain=gains), lambda: drf.qk_norm_rope(q, k, "rms", q_bias=gains), lambda: drf.block_select(q, k[:1], 32, 32, 1),
                     lambda: drf.block_select(q, k, 48, 32, 1), lambda: drf.block_select(q, k, 32, 32, 0), lambda: drf.block_select(q, k[:, :, :3], 32, 32, 1),
                     lambda: drf.block_attention(q, k, v, words[..., :0], 32, 32), lambda: drf.block_attention(q, k, v, words, 64, 32), lambda: drf.block_attention(q, k, f, words, 32, 32),
                     lambda: drf.block_attention(q, k, v, words, 32, 32, scale=-1.0), lambda: drf.block_attention(q, k, v.contiguous()[:, 1:], words, 32, 32)):
            with pytest.raises((AssertionError, ValueError, drf.DrfError)) as e:
                call()
            bad.append((type(e.value), e.value.status if isinstance(e.value, drf.DrfError) else None))
        got.append((out, bad))
    assert all(torch.equal(a, b) for a, b in zip(got[0][0], got[1][0])) and got[0][1] == got[1][1]
