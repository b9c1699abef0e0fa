"""What the tests of the operators around a block's Linears compare with, by itself: a wrong result is refused whatever it is."""
import numpy as np
import pytest

from test_gpu_block_operator_values import close
from test_host_block_operators import EINVAL, norm, residual

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
