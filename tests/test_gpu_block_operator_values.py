"""The operators around a block's Linears at the ends of their values: rows of any magnitude through the norms.  References are those of test_gpu_block_operators.py, and so
are the tolerances; a result that is no number is refused wherever the reference has one."""
import numpy as np
import pytest

from test_gpu_block_operators import HALF, f64, normed, rand
from test_gpu_block_operators import drf, torch  # noqa: F401

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
