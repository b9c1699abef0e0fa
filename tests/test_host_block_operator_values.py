"""What the tests of the operators around a block's Linears compare with, by itself: a wrong result is refused whatever it is."""
import numpy as np
import pytest

from test_gpu_block_operator_values import close
from test_host_block_operators import EINVAL, FAKE, adapters, ffn, norm, residual, rows

from paper_2603_25872_amd import drf


def test_results_that_are_no_numbers_are_refused():
    want = np.array([[1.0, -2.0], [np.inf, np.nan]])
    close(want.copy(), want, "f32", 0.0)
    for bad in (np.nan, np.inf, -np.inf, 1.0 + 2.0 ** -20, -1.0):
        got = want.copy()
        got[0, 0] = bad
        for slack in (0.0, np.zeros((2, 2)), 2.0 ** -21):
            with pytest.raises(AssertionError):
                close(got, want, "f32", slack)
    for at, bad in (((1, 0), 3.0), ((1, 0), -np.inf), ((1, 0), np.nan), ((1, 1), 0.0), ((1, 1), np.inf)):
        got = want.copy()
        got[at] = bad
        with pytest.raises(AssertionError):
            close(got, want, "f32", 1.0)
    with pytest.raises(AssertionError):
        close(want[:1], want, "f32", 0.0)


def test_a_residual_update_without_a_branch_has_no_look_at_its_arguments():
    for over in (dict(y_scale=float("nan")), dict(y_scale=float("inf")), dict(after=norm(3)), dict(after=norm(eps=-1.0)), dict(after=norm(drf.QK_NONE, 0.0, 0x10000)),
                 dict(after=norm(drf.QK_RMS, 0.0, None, 0x10000))):
        assert residual(y=None, out=None, slots=0, **over) == 0
        assert residual(slots=0, **over) == EINVAL


def lie_on_one_another(slots, tokens, width, ss, ts):
    at = np.sort((ss * np.arange(slots)[:, None] + ts * np.arange(tokens)).ravel())
    return bool((np.diff(at) < width).any())


def test_outputs_whose_rows_lie_on_one_another_in_any_way_are_refused():
    """Windows over one another, rows between rows: as their addresses are.  What lies right is refused for the next reason there is, that the output is an input's."""
    rng = np.random.default_rng(0)
    seen = [0, 0]
    cases = [(2, 64, 64, 64, 64), (3, 5, 64, 64, 128), (5, 3, 64, 128, 64), (4, 6, 64, 64, 256), (7, 9, 1, 9, 1), (7, 9, 1, 1, 7), (7, 9, 1, 8, 1), (2, 64, 64, 2 ** 40, 64), (64, 2, 64, 64, 2 ** 40)]
    cases += [tuple(int(v) for v in (*rng.integers(1, 12, 2), rng.integers(1, 20), *(rng.integers(0, 60, 2) if k % 2 else rng.integers(0, 400, 2)))) for k in range(4000)]
    for slots, tokens, width, ss, ts in cases:
        bad = lie_on_one_another(slots, tokens, width, ss, ts)
        seen[bad] += 1
        for sign in ((1, 1), (-1, 1), (1, -1)):
            t = rows(2 * FAKE, ss * sign[0], ts * sign[1])
            assert residual(slots=slots, tokens=tokens, width=width, h=None, out=t, x=rows(FAKE, 400, 20)) == EINVAL
            text = drf.lib().drf_last_error()
            assert (b"lie on one another" in text) == bad and (bad or b"lies on another tensor" in text), (slots, tokens, width, ss, ts)
        for call in (ffn, adapters):
            if ts < 2 ** 22:
                assert call(dtype=drf.F32, slots=slots, tokens=tokens, out_width=width, out=rows(FAKE, ss, ts)) == EINVAL
                text = drf.lib().drf_last_error()
                assert (b"lie on one another" in text) == bad and (bad or b"lies on the input" in text), (call, slots, tokens, width, ss, ts)
    assert min(seen) > 400
    # (the longest pass there is: 2^15 of both)
    assert residual(slots=2 ** 15, tokens=2 ** 15, width=1, h=None, out=rows(2 * FAKE, 2 ** 15 + 2, 2 ** 15 + 1)) == EINVAL
    assert b"lies on another tensor" in drf.lib().drf_last_error()
