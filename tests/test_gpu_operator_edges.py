"""The attention operators at the edges of what their calls allow, against their definitions in float64.

Tolerances beyond those of test_gpu_operators.py stand at their tests; a rounding is off by at most half a step, 2^-8 of the value in bf16 and 2^-24 in
fp32."""
import numpy as np
import pytest

import test_gpu_operators as ops
from paper_2603_25872_amd import drf as D_

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available()
    return t


@pytest.fixture(scope="module")
def drf():
    D_.lib()
    return D_


# ---- rotations ------------------------------------------------------------------------------------------


def same_bits(torch, a, b):
    """Equal bit for bit, one NaN as good as another."""
    as_int = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
    nan = torch.isnan(b)
    return torch.equal(torch.isnan(a), nan) and torch.equal(a.contiguous().view(as_int)[~nan], b.contiguous().view(as_int)[~nan])


UNTURNED = [((24,), "halves"), ((32, 8), "halves"), ((36,), "halves"), ((6, 10), "halves"), ((24,), "pairs"), ((36, 4), "pairs"), ((0, 0), "pairs")]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dims,kind", UNTURNED)
@pytest.mark.parametrize("layout", ["plain", "heads", "odd"])
def test_columns_that_do_not_turn_are_left_as_they_are(torch, drf, dtype, dims, kind, layout):
    """Infinities, NaN, zeros of both signs and the largest numbers among the columns behind the sections, on 16-byte and element accesses: bit for bit the
    input's (a power of two times it for the queries with a scale), and nothing of them in the columns that turn."""
    S, N, H, d, at = 2, 13, 5, 72, sum(dims)
    rng = np.random.default_rng(at)
    x, v = ops.tensor(torch, rng, (S, N, H, d), dtype, layout)
    special = torch.tensor([float("inf"), float("-inf"), float("nan"), -0.0, 0.0, 1e38, -1e38, 1.5], device="cuda").to(x.dtype)
    x[..., at:] = special[torch.from_numpy(rng.integers(0, 8, (S, N, H, d - at))).cuda()]
    cfg = drf.rope_config(dims, (1, 4)[2 - len(dims):], layout=kind, origin=(5,) * len(dims))
    want = ops.rotated(v, cfg)
    lens = torch.tensor([N, 4], dtype=torch.int32, device="cuda")
    for got, length in ((drf.rope(x, cfg), N), (drf.rope(x, cfg, lens=lens), 4), (drf.qk_norm_rope(x, x, "none", cfg, q_scale=0.5)[1], N)):
        assert same_bits(torch, got[..., at:], x[..., at:])
        ops.check(got[1, :length, :, :at], want[1, :length, :, :at], dtype, 2.0 ** -19 * np.abs(v).max())
    assert same_bits(torch, drf.qk_norm_rope(x, x, "none", cfg, q_scale=0.5)[0][..., at:], (x * 0.5)[..., at:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dims,kind", UNTURNED)
@pytest.mark.parametrize("layout", ["plain", "odd"])
def test_infinite_parameters_of_columns_that_do_not_turn(torch, drf, dtype, dims, kind, layout):
    """A gain and a bias that are infinite reach their own columns alone."""
    S, N, H, d, at = 1, 9, 3, 72, sum(dims)
    rng = np.random.default_rng(at + 1)
    x, v = ops.tensor(torch, rng, (S, N, H, d), dtype, layout)
    gain, bias = rng.uniform(0.5, 2, d).astype(np.float32), rng.uniform(-1, 1, d).astype(np.float32)
    gain[at + 1], bias[at + 4] = np.inf, -np.inf
    cfg = drf.rope_config(dims, (1, 4)[2 - len(dims):], layout=kind)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    for norm, b in (("rms", None), ("layer", bias)):
        y = ops.normed(v, norm, gain, b, 1e-6)
        got = drf.qk_norm_rope(x, x, norm, cfg, dev(gain), dev(gain), None if b is None else dev(b), None if b is None else dev(b))
        fine = np.isfinite(y)
        for g in got:
            g = g.double().cpu().numpy()
            assert np.array_equal(g[~fine], y[~fine])
            want = ops.rotated(np.where(fine, y, 0.0), cfg)
            ops.check(torch.from_numpy(np.where(fine, g, 0.0)), want, dtype, 2.0 ** -19 * np.abs(want).max())


# ---- which blocks ---------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [8, 64, 100, 128])
@pytest.mark.parametrize("M,kv_block", [(3 * 64 + 37, 64), (70 * 32 + 31, 32), (2 * 128 + 1, 128)])
def test_equal_keys_tie_in_a_block_that_is_not_full(torch, drf, dtype, d, M, kv_block):
    """Every key row the same, of any values: every block has the same mean and score, the last one too that holds fewer rows (its sum of up to 128
    equal fp32 rows is exact in 64 bits, and so is the mean), so the lowest blocks are chosen."""
    rng = np.random.default_rng(d + M)
    H, nk = 4, -(-M // kv_block)
    for _ in range(12):
        q, _ = ops.tensor(torch, rng, (1, 150, H, d), dtype, "plain")
        k, _ = ops.tensor(torch, rng, (1, 1, H, d), dtype, "plain")
        for topk in (1, 2, nk - 1):
            got = ops.bits(torch, drf.block_select(q, k.expand(1, M, H, d), 32, kv_block, topk), nk)
            assert np.array_equal(got, np.broadcast_to(np.arange(nk) < topk, got.shape)), topk


# ---- attention ------------------------------------------------------------------------------------------


FORMS = [("f32", 1), ("bf16", 1)] + [("bf16", t) for t in ops.TILES]


def weighted_alike(torch, drf, dtype, q, k, v, mask, weighted, q_block, kv_block, tiles, scale):
    """Attention whose weights are all alike over the keys `weighted` [tokens] of a list and zero over the others; where a list has none of them, over all its
    keys.  What is left is the sum of as many values in fp32, 2^-24 of the mean of |v| for each at most, and in bf16 the weights' own rounding, half a step: they are alike
    but need not be one (a power of two of any fraction, by what they are taken relative to), and the denominator sums them before it at widths of 32."""
    S, N, H, d = q.shape
    M = k.shape[1]
    c = -(-tiles // (-(-N // 32) * H * S))
    got = drf.block_attention(q.repeat(c, 1, 1, 1), k.repeat(c, 1, 1, 1), v.repeat(c, 1, 1, 1), ops.pack(torch, mask).repeat(c, 1, 1, 1), q_block, kv_block, scale)
    vv = v.double().cpu().numpy()
    want, mag = np.zeros((S, N, H, d)), np.zeros((S, N, H, d))
    for h in range(H):
        for i in range(mask.shape[2]):
            keys = np.flatnonzero(np.repeat(mask[0, h, i], kv_block)[:M])
            keys = keys[weighted[keys]] if weighted[keys].any() else keys
            if keys.size:
                want[0, i * q_block:(i + 1) * q_block, h] = vv[0, keys, h].mean(0)
                mag[0, i * q_block:(i + 1) * q_block, h] = np.abs(vv[0, keys, h]).mean(0)
    ops.check(got[:1], want, dtype, (M + 4) * 2.0 ** -24 * mag + (ops.HALF["bf16"] * np.abs(want) if dtype == "bf16" else 0.0))
    assert (got == got[:1]).all()


@pytest.mark.parametrize("dtype,tiles", FORMS)
@pytest.mark.parametrize("d", [24, 64, 72, 128])
@pytest.mark.parametrize("qb", [64, 128])
@pytest.mark.parametrize("scale", [1e-20, 2e-38, 1e-38, 1e-42])
def test_the_smallest_scales(torch, drf, dtype, tiles, d, qb, scale):
    """Scores that the scale takes all difference from: the mean of the values."""
    rng = np.random.default_rng(d)
    (q, _), (k, _), (v, _) = (ops.tensor(torch, rng, (1, n, 2, d), dtype, "plain") for n in (96, 160, 160))
    mask = ops.random_mask(rng, 1, 2, 96, 160, qb, 32, 0.7)
    weighted_alike(torch, drf, dtype, q, k, v, mask, np.ones(160, bool), qb, 32, tiles, scale)


@pytest.mark.parametrize("dtype,tiles", FORMS)
@pytest.mark.parametrize("d", [24, 64, 72, 128])
@pytest.mark.parametrize("qb", [64, 128])
@pytest.mark.parametrize("scale", [1e-37, 0.125, 1.0, 30.0, 1e6])
@pytest.mark.parametrize("value", [-3.3895313892515355e38, 3.3895313892515355e38])
def test_scores_as_large_as_the_type_has(torch, drf, dtype, tiles, d, qb, scale, value):
    """Keys that a column of them marks with the type's lowest value have no weight beside others and equal weights among themselves; with its
    largest they have all of it (e^-33 is left at the smallest scale here).  Marked first, last, all and none."""
    rng = np.random.default_rng(d)
    N, M = 96, 160
    (q, _), (k, _), (v, _) = (ops.tensor(torch, rng, (1, n, 2, d), dtype, "plain") for n in (N, M, M))
    q.zero_()
    q[..., 0] = 1.0
    for marked in (np.arange(M) < 64, np.arange(M) >= 100, np.ones(M, bool), np.zeros(M, bool), rng.random(M) < 0.3):
        k[..., 0] = torch.from_numpy(np.where(marked, value, 0.0)).to(k).view(1, M, 1)
        mask = ops.random_mask(rng, 1, 2, N, M, qb, 32, 0.7)
        mask[0, 0, 0, :3] = [1, 0, 1]
        weighted_alike(torch, drf, dtype, q, k, v, mask, marked if value > 0 else ~marked, qb, 32, tiles, scale)


def test_the_smallest_scales_and_largest_scores_in_parts(torch, drf):
    """The same where several workgroups share a list."""
    rng = np.random.default_rng(0)
    M, d = 8192, 64
    (q, _), (k, _), (v, _) = (ops.tensor(torch, rng, (1, n, 2, d), "bf16", "plain") for n in (3, M, M))
    words = ops.pack(torch, np.ones((1, 2, 1, M // 64), bool))
    vv = v.double().cpu().numpy()
    ops.check(drf.block_attention(q, k, v, words, 32, 64, 1e-39, split=True), np.broadcast_to(vv.mean(1, keepdims=True), q.shape), "bf16", (M + 4) * 2.0 ** -24 * np.abs(vv).mean(1, keepdims=True))
    q.zero_()
    q[..., 0] = 1.0
    for weighted, value in ((np.arange(M) >= 7000, -3.3895313892515355e38), (np.arange(M) == 4321, 3.3895313892515355e38)):
        k[..., 0] = torch.from_numpy(np.where(weighted == (value > 0), value, 0.0)).to(k).view(1, M, 1)
        want, mag = vv[:, weighted].mean(1, keepdims=True), np.abs(vv[:, weighted]).mean(1, keepdims=True)
        ops.check(drf.block_attention(q, k, v, words, 32, 64, 1.0, split=True), np.broadcast_to(want, q.shape), "bf16", (M + 4) * 2.0 ** -24 * mag)


def test_rotation_of_more_rows_than_one_launch_takes(torch, drf):
    """34 GB of rows in place, as 16-byte accesses: each turns once, by its own position."""
    d, tokens = 128, 8 * 2 ** 23 + 13
    if torch.cuda.mem_get_info()[0] < 60 * 2 ** 30:
        pytest.skip("needs 60 GB")
    x = torch.ones(1, tokens, 1, d, device="cuda")
    drf.rope(x, drf.rope_config((2,), (1,), theta=1.0), out=x)
    for a in range(0, tokens, 2 ** 22):
        part = x[0, a:a + 2 ** 22, 0]
        phi = torch.arange(a, a + part.shape[0], device="cuda", dtype=torch.float64)
        want = torch.stack([phi.cos() - phi.sin(), phi.sin() + phi.cos()], 1)
        assert (part[:, :2] - want).abs().max() <= 2.0 ** -19 and (part[:, 2:] == 1).all()
    del x, part
    torch.cuda.empty_cache()


# ---- layouts --------------------------------------------------------------------------------------------


def with_odd_unused_strides(torch, x):
    """The same memory with strides that no multiple of 16 bytes is, where a dimension has one element."""
    strides = [s if n > 1 else 2 ** 24 + 3 for n, s in zip(x.shape[:3], x.stride())]
    return torch.as_strided(x, x.shape, (*strides, 1), x.storage_offset())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,N,M,H,Hk", [(1, 1, 100, 1, 1), (1, 40, 100, 2, 1), (2, 1, 1, 2, 2), (1, 1, 1, 4, 1), (2, 33, 33, 1, 1)])
def test_strides_of_one_element_are_not_used(torch, drf, dtype, S, N, M, H, Hk):
    rng = np.random.default_rng(N)
    d = 64
    q, k, v = (ops.tensor(torch, rng, (S, n, h, d), dtype, "plain")[0] for n, h in ((N, H), (M, Hk), (M, Hk)))
    cfg, odd = drf.rope_config((32, 32), (1, 9)), lambda t: with_odd_unused_strides(torch, t)  # noqa: E731
    words = drf.block_select(q, k, 32, 32, 2)
    assert torch.equal(drf.block_select(odd(q), odd(k), 32, 32, 2), words)
    assert torch.equal(drf.rope(odd(q), cfg, out=odd(torch.empty_like(q))), drf.rope(q, cfg))
    if N == M:
        got = drf.qk_norm_rope(odd(q), odd(k), "rms", cfg, q_out=odd(torch.empty_like(q)), k_out=odd(torch.empty_like(k)))
        assert all(torch.equal(a, b) for a, b in zip(got, drf.qk_norm_rope(q, k, "rms", cfg)))
    want = drf.block_attention(q, k, v, words, 32, 32)
    assert torch.equal(drf.block_attention(odd(q), odd(k), odd(v), words, 32, 32, out=odd(torch.empty_like(q))), want)
    same = odd(q.clone())
    assert torch.equal(drf.rope(same, cfg, out=torch.as_strided(same, q.shape, q.stride())), drf.rope(q, cfg))      # in place


@pytest.mark.parametrize("layout", ["plain", "odd"])
@pytest.mark.parametrize("kind", ["pairs", "halves"])
def test_angles_are_right_where_a_sine_or_cosine_is_small(torch, drf, layout, kind):
    """(1, 0) turns to the cosine and sine of the angle.  A position below 4096 is at most 652 turns, of which double precision keeps 652 2^-51 (frequency, product,
    rest), 2 pi times that together with the oracle's own below 2^-37 rad.  The rest of a quarter turn is rounded to fp32, half a step, of which sine and cosine
    have at most as much; each of them is off by at most 4 steps of 2^-23; the products with 1 and 0 are exact."""
    rng = np.random.default_rng(3)
    S, N, H, d, dims = 1, 3000, 1, 64, (40, 24)
    cfg = drf.rope_config(dims, (1, 1), layout=kind)
    x, v = ops.tensor(torch, rng, (S, N, H, d), "f32", layout, 0.0)
    _, first, second = ops.angles(cfg, S, N)
    x[..., torch.from_numpy(first).cuda()] = 1.0
    p = np.where(rng.random((N, 2)) < 0.5, rng.integers(-4096, 4096, (N, 2)), rng.uniform(-40, 40, (N, 2))).astype(np.float32)
    phi, _, _ = ops.angles(cfg, S, N, p)
    got = drf.rope(x, cfg, positions=torch.from_numpy(p).cuda()).double().cpu().numpy()[:, :, 0]
    for columns, want in ((first, np.cos(phi)), (second, np.sin(phi))):
        off = np.abs(got[..., columns] - want)
        assert (off <= (2.0 ** -24 + 4 * 2.0 ** -23) * np.abs(want) + 2.0 ** -37).all(), float((off / np.abs(want)).max() * 2.0 ** 23)


def test_scratch_that_a_call_has_no_use_for_is_not_looked_at(torch, drf):
    """Where drf_block_attention_scratch_bytes() is 0, the call with scratch, of any size and alignment, is the one without."""
    torch.manual_seed(0)
    for dtype, kind in ((torch.bfloat16, drf.BF16), (torch.float32, drf.F32)):
        q, k, v = (torch.randn(1, n, 2, 64, device="cuda").to(dtype) for n in (5, 300, 300))
        words, out = drf.block_select(q, k, 32, 32, 3), torch.empty_like(q)
        shape = drf.AttnShape(kind, 1, 5, 300, 2, 2, 64, None, None)
        assert drf.lib().drf_block_attention_scratch_bytes(drf.C.byref(shape)) == 0
        scratch = torch.empty(16, device="cuda")
        rc = drf.lib().drf_block_attention_split(drf.C.byref(shape), 32, 32, 0.125, words.data_ptr(), *[drf.C.byref(drf._heads(t)) for t in (q, k, v, out)],
                                                 scratch.data_ptr() + 4, 0, drf._current(q))
        assert rc == 0 and torch.equal(out, drf.block_attention(q, k, v, words, 32, 32, scale=0.125))


@pytest.mark.parametrize("dtype,S,N,M,H,Hk,d,kv_block,share,split", [
    ("bf16", 1, 1, 20000, 2, 1, 128, 32, 0.7, True), ("bf16", 1, 33, 14000, 2, 2, 64, 32, 0.3, True), ("bf16", 1, 1, 9000, 16, 2, 72, 128, 1.0, True),
    ("bf16", 1, 5, 8255, 1, 1, 128, 64, 0.05, True), ("bf16", 2, 64, 16384, 1, 1, 96, 128, 0.4, True), ("bf16", 1, 1, 9001, 2, 1, 64, 32, 1.0, False),
    ("bf16", 1, 33, 5000, 2, 1, 128, 64, 0.4, False), ("bf16", 4, 300, 3001, 16, 1, 72, 32, 0.3, False), ("bf16", 4, 700, 3001, 16, 1, 128, 64, 0.5, False),
    ("bf16", 2, 700, 3001, 32, 1, 128, 128, 0.5, False), ("f32", 1, 1, 9001, 2, 1, 128, 32, 0.6, False), ("f32", 2, 70, 4000, 2, 1, 64, 64, 1.0, False)])
def test_every_step_of_a_list_counts_once(torch, drf, dtype, S, N, M, H, Hk, d, kv_block, share, split):
    """Queries of zeros weigh the keys of a list alike, and column c of the values is one on the 32 keys of one step alone: the result is that step's share of the
    list, nothing if a step is missed, twice as much if it is taken twice.  Every step of the keys is a column's in turn.  Weights and sums are whole numbers,
    exact in fp32; the quotient and product with its inverse are off by 2^-22."""
    rng = np.random.default_rng(M + d)
    q_block = 128 if N == 700 and kv_block == 128 else 64 if N > 64 else 32
    mask = ops.random_mask(rng, S, H, N, M, q_block, kv_block, share)
    q, k = torch.zeros(S, N, H, d, device="cuda"), torch.randn(S, M, Hk, d, device="cuda")
    chosen = np.repeat(mask, kv_block, axis=-1)[..., :M]                        # [slots, heads, query blocks, keys]
    steps = -(-M // 32)
    a_step = np.add.reduceat(chosen, np.arange(0, M, 32), axis=-1, dtype=np.int64)
    share_of = a_step / np.maximum(chosen.sum(-1, keepdims=True), 1)            # [slots, heads, query blocks, steps]
    q, k, words = q.to(ops.dtype_of(torch, dtype)), k.to(ops.dtype_of(torch, dtype)), ops.pack(torch, mask)
    step_of = torch.arange(M, device="cuda") // 32
    row_block = np.arange(N) // q_block
    for first in range(0, steps, d):
        v = (step_of[:, None] == first + torch.arange(d, device="cuda")).to(q.dtype).view(1, M, 1, d).expand(S, M, Hk, d).contiguous()
        got = drf.block_attention(q, k, v, words, q_block, kv_block, split=split)
        want = np.zeros((S, H, len(row_block), d))
        want[..., :min(d, steps - first)] = share_of[:, :, row_block, first:first + d]
        want = want.transpose(0, 2, 1, 3)
        ops.check(got, want, dtype, 2.0 ** -22 * want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_expanded_inputs_and_outputs(torch, drf, dtype):
    """Tensors expanded over slots, tokens or heads are inputs like others; as outputs they are refused."""
    rng = np.random.default_rng(9)
    S, N, H, d = 2, 33, 3, 64
    cfg = drf.rope_config((32, 32), (1, 9))
    for size in ((1, N, H, d), (S, 1, H, d), (S, N, 1, d)):
        x, v = ops.tensor(torch, rng, size, dtype, "plain")
        wide, v = x.expand(S, N, H, d), np.broadcast_to(v, (S, N, H, d))
        whole = wide.contiguous()
        ops.check(drf.rope(wide, cfg), ops.rotated(v, cfg), dtype, 2.0 ** -19 * np.abs(v).max())
        words = drf.block_select(wide, wide, 32, 32, 1)
        assert torch.equal(words, drf.block_select(whole, whole, 32, 32, 1))
        assert torch.equal(drf.block_attention(wide, wide, wide, words, 32, 32), drf.block_attention(whole, whole, whole, words, 32, 32))
        for call in (lambda: drf.rope(whole, cfg, out=wide), lambda: drf.qk_norm_rope(whole, whole, "rms", cfg, k_out=wide),
                     lambda: drf.block_attention(whole, whole, whole, words, 32, 32, out=wide)):
            with pytest.raises(drf.DrfError):
                call()


def test_results_are_unknown_to_autograd(torch, drf):
    """Of inputs that require gradients too: no result carries a gradient that is not the operator's."""
    x = torch.randn(2, 40, 2, 64, device="cuda", requires_grad=True)
    lens, cfg = torch.tensor([40, 7], dtype=torch.int32, device="cuda"), drf.rope_config((32, 32), (1, 9))
    for n in (None, lens):
        words = drf.block_select(x, x, 32, 32, 1, q_lens=n, kv_lens=n)
        out = [drf.rope(x, cfg, lens=n), *drf.qk_norm_rope(x, x, "rms", cfg, lens=n), drf.block_attention(x, x, x, words, 32, 32, q_lens=n, kv_lens=n)]
        assert not any(t.requires_grad for t in out)
        assert torch.equal(out[0], drf.rope(x.detach(), cfg, lens=n))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["plain", "odd"])
@pytest.mark.parametrize("eps", [1e-300, 1e-46, 1e-30, 1e30])
def test_norms_of_rows_of_zeros(torch, drf, dtype, layout, eps):
    """Zeros over the root of any eps above zero are zeros, biases stay; the rows beside them are what they are."""
    rng = np.random.default_rng(12)
    x, v = ops.tensor(torch, rng, (1, 9, 3, 40), dtype, layout)
    x[:, ::2] = 0.0
    v[:, ::2] = 0.0
    bias = rng.uniform(-1, 1, 40).astype(np.float32)
    for norm, b in (("rms", None), ("layer", bias)):
        want = ops.normed(v, norm, None, b, eps)
        dev = None if b is None else torch.from_numpy(b).cuda()
        for got in drf.qk_norm_rope(x, x, norm, q_bias=dev, k_bias=dev, eps=eps):
            ops.check(got, want, dtype, 2.0 ** -19 * np.abs(want).max())
