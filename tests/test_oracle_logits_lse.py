"""The oracle's log-sum-exp of a student's row: of the logits alone, as include/msd.h has it."""
import numpy as np
import pytest

from oracle import logits as O

INF = np.inf


@pytest.mark.parametrize("ids", [[0, 2], [-1, -1]], ids=["entries", "none"])
@pytest.mark.parametrize("values", [[1.0, 0.5], [-INF, -INF], [np.nan, 0.0]], ids=str)
def test_log_sum_exp_of_a_students_row(ids, values):
    def lse(row, T=2.0):
        return O.distill(np.array(row), ids, values, T)[1]
    assert abs(lse([2.0, 2.0, -INF, 2.0]) - (1 + np.log(3))) < 1e-15
    assert lse([-INF] * 4) == -INF and lse([-INF] * 4, 1e6) == -INF
    assert np.isnan(lse([0.0, np.nan, 1.0, -INF])) and np.isnan(lse([np.nan] * 4))
    assert np.isnan(lse([0.0, INF, 1.0, -INF]))


def test_loss_and_gradient_of_a_row_of_minus_infinity():
    row = np.full(5, -INF)
    loss, _, dx, _, _ = O.distill(row, [0, 3], [1.0, 2.0], 1.0)
    assert np.isnan(loss) and np.isnan(dx).all()
    loss, _, dx, _, _ = O.distill(row, [-1, 5], [1.0, 2.0], 1.0)
    assert loss == 0 and (dx == 0).all()
