"""The operators around a block's Linears where their indices are largest: tensors whose offsets pass 32 bits, more rows than one launch takes; and calls that meet: from
two threads, as a process's first inside a capture.  References and tolerances are those of test_gpu_block_operators.py."""
import os
import subprocess
import sys
import threading

import numpy as np
import pytest

from test_gpu_block_operators import D_, adapted, adapter_case, check, dtype_of, f64, ffn, ffn_case, rand, residual, run_adapters  # noqa: F401
from test_gpu_block_operators import drf, forced, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def give_back(torch):  # noqa: F811
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def far(torch, shape, strides, dtype):  # noqa: F811
    """A tensor of those strides, by itself in as much memory as they take."""
    n = sum((k - 1) * s for k, s in zip(shape, strides)) + shape[-1]
    return torch.empty(n, dtype=dtype, device="cuda").as_strided(shape, (*strides, 1))


# (slots, tokens, stride of a slot, stride of a token): a slot beyond 4 GiB from the next, 300 rows of the widest spread, 90 short slots that one tile crosses
FAR = [(3, 40, 2 ** 31 + 8, 200), (1, 300, 0, 2 ** 22 - 8), (90, 3, 2 ** 23 + 8, 2 ** 21 + 8)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,N,ss,ts", FAR)
def test_offsets_past_32_bits(torch, drf, forced, dtype, S, N, ss, ts):  # noqa: F811
    rng = np.random.default_rng(N)
    x, w_in, w_out, b_in, b_out = ffn_case(torch, rng, S, N, 136, 64, 136, dtype)
    _, w, a, b, which, bias, scales = adapter_case(torch, rng, S, N, 136, 136, 40, 3, dtype)
    block, low = ffn(f64(x), f64(w_in), f64(w_out), f64(b_in), f64(b_out), "silu", dtype), adapted(f64(x), f64(w), f64(a), f64(b), which, f64(bias), f64(scales), dtype)
    wide, out = far(torch, x.shape, (ss, ts), x.dtype).copy_(x), far(torch, x.shape, (ss, ts), x.dtype)
    for tile in (-1, 0, 1, 2, 3, 5, 6, 7, 9, 10, 13, 14):
        forced(tile)
        out.fill_(7.0)
        check(drf.gated_ffn(wide, w_in, w_out, b_in, b_out, out=out), block[0], dtype, block[1])
        out.fill_(7.0)
        check(run_adapters(torch, drf, wide, w, a, b, which, bias, scales, out=out), low[0], dtype, low[1])
    gate = rand(torch, rng, (S, 136))
    args = dict(gate=gate, after="rms", after_gain=None, after_bias=None, x_scale=0.5, y_scale=1.0, before="layer", before_gain=None, before_bias=None, shift=None, scale=None, eps=1e-5)
    z, ez, h, eh = residual(f64(x), f64(x), {**args, "gate": f64(gate)})
    got = drf.residual_norm(wide, x, out=wide, h_out=out, **args)
    check(got[0], z, dtype, ez)
    check(got[1], h, dtype, eh)


@pytest.mark.parametrize("dtype,tiles,S,D,F", [("bf16", (4, 5, 8, 10, 12, 13), 65540, 8, 8), ("f32", (8, 14), 131080, 4, 1)])
def test_more_tiles_than_one_launch_takes(torch, drf, forced, dtype, tiles, S, D, F):  # noqa: F811
    """One slot's rows for all slots: all results are the first slot's."""
    rng = np.random.default_rng(S)
    N = 4099
    x, w_in, w_out, b_in, b_out = ffn_case(torch, rng, 1, N, D, F, 1, dtype)
    want, slack = ffn(f64(x), f64(w_in), f64(w_out), f64(b_in), f64(b_out), "silu", dtype)
    for tile in tiles:
        forced(tile)
        got = drf.gated_ffn(x.expand(S, N, D), w_in, w_out, b_in, b_out)
        check(got[:1], want, dtype, slack)
        assert (got == got[:1]).all(), tile
        del got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_slots_than_one_launch_takes(torch, drf, dtype):  # noqa: F811
    rng = np.random.default_rng(5)
    S = 2 ** 22 + 72
    x, w, a, b, _, bias, scales = adapter_case(torch, rng, 1, 1, 8, 8, 8, 3, dtype)
    which = [-1, 0, 1, 2]
    want, slack = adapted(f64(x.expand(4, 1, 8)), f64(w), f64(a), f64(b), which, f64(bias), f64(scales), dtype)
    got = drf.linear_adapters(x.expand(S, 1, 8), w, a, b, torch.tensor(which, dtype=torch.int32, device="cuda").repeat(S // 4), bias, scales)
    check(got[:4], want, dtype, slack)
    assert (got.view(S // 4, 4, 8) == got[:4, 0]).all()


@pytest.mark.parametrize("dtype,S,D,per_token", [("bf16", 2 ** 19 + 9, 8, False), ("bf16", 2 ** 19 + 9, 8, True), ("f32", 2 ** 19 + 9, 4, True), ("f32", 2 ** 19 + 9, 3, False), ("bf16", 2 ** 16 + 3, 2050, False)])
def test_more_rows_than_one_launch_takes(torch, drf, dtype, S, D, per_token):  # noqa: F811
    """Rows of a wave each, of waves that share a slot's modulation and of a workgroup each; one slot's rows for all slots."""
    rng = np.random.default_rng(D)
    N = 64
    x, shift = rand(torch, rng, (1, N, D), dtype), rand(torch, rng, (1, N, D) if per_token else (1, D))
    args = dict(gate=None, after="none", after_gain=None, after_bias=None, x_scale=0.5, y_scale=1.0, before="layer", before_gain=None, before_bias=None, scale=None, eps=1e-2)
    want, slack = residual(f64(x), None, {**args, "shift": f64(shift)})[2:]
    got = drf.residual_norm(x.expand(S, N, D), shift=shift.expand(S, *shift.shape[1:]), **args)[1]
    check(got[:1], want, dtype, slack)
    assert (got == got[:1]).all()


def test_from_two_threads(torch, drf):  # noqa: F811
    """Calls of two threads on streams of their own, through the same kernels with other sizes."""
    rng = np.random.default_rng(3)
    sides = []
    for S, N in ((2, 300), (5, 77)):
        c = ffn_case(torch, rng, S, N, 136, 264, 136, "bf16")
        sides.append((c, adapter_case(torch, rng, S, N, 136, 136, 24, 3, "bf16")))
    run = lambda c, d: [t for _ in range(40) for t in (drf.gated_ffn(*c), run_adapters(torch, drf, *d), drf.residual_norm(c[0], d[0])[1])]  # noqa: E731
    want = [run(*s) for s in sides]
    torch.cuda.synchronize()
    got, failed = [None, None], []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                got[i] = run(*sides[i])
                torch.cuda.current_stream().synchronize()
        except Exception as e:
            failed.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    for p, q in zip(got, want):
        assert all(torch.equal(s, t) for s, t in zip(p, q))


FIRST = """
import torch
from paper_2603_25872_amd import drf
torch.manual_seed(1)
r = lambda *s: torch.randn(*s, device="cuda").bfloat16()
x, y, w, w_out, a, b, which = r(3, 700, 256), r(3, 700, 256), r(1024, 256), r(256, 512), r(2, 16, 256), r(2, 1024, 16), torch.tensor([1, -1, 0], dtype=torch.int32, device="cuda")
call = lambda: (*drf.residual_norm(x, y, before="rms"), drf.gated_ffn(x, w, w_out), drf.gated_ffn(x[:1, :1], w, w_out), drf.linear_adapters(x, w, a, b, which))
g = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(g):
    got = call()
for k in range(3):
    x.copy_(r(3, 700, 256))
    want = call()
    torch.cuda.synchronize()
    for t in got:
        t.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(s, t) for s, t in zip(got, want)), k
print("replays agree")
"""


def test_first_calls_of_a_process_are_captured():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST], cwd=root, capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and "replays agree" in r.stdout, r.stdout + r.stderr
