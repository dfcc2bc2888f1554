"""The rest of a top-log-probability list in the oracle: exact where one entry has nearly all of the
probability, and none only where the student has none either."""
from fractions import Fraction

import numpy as np
import pytest

from oracle.logprobs import topk_ce


@pytest.mark.parametrize("left", [1e-3, 1e-5, 1e-7, 1e-9])
def test_a_small_rest_is_exact(left):
    """Probabilities 1 - left, left / 2, left / 4: a quarter of `left` is outside."""
    ids = np.array([[4, 1, 6]])
    lp = np.array([[np.log1p(-left), np.log(left / 2), np.log(left / 4)]])
    x = np.zeros((1, 8))
    x[0, 4] = 3.0
    _, pairs, grad = topk_ce(ids, lp, x, [0], [0])
    q = np.exp(x[0]) / np.exp(x[0]).sum()
    outside = [0, 2, 3, 5, 7]
    q_rest = q[outside].sum()
    rest = float(Fraction(left) / 4)
    others = -(np.exp(lp[0]) * np.log(q[[4, 1, 6]])).sum()
    assert np.isclose(pairs[0], others - rest * np.log(q_rest), rtol=1e-15)
    # what the rest takes from each element outside, to 8 digits of itself
    taken = q[outside] - grad[0, outside]
    assert np.allclose(taken, rest * q[outside] / q_rest, rtol=1e-8 + 1e-15 / rest, atol=0)


def test_no_rest_where_neither_has_one():
    ids = np.array([[0, 1, -1]])
    x = np.array([[1.0, 2.0, -np.inf, -np.inf], [1.0, 2.0, 0.0, -np.inf], [1.0, 2.0, -1e4, -np.inf]])
    for short, counted in ((3e-7, (False, True, False)), (2e-6, (True, True, True))):
        lp = np.array([[np.log(0.5), np.log(0.5 - short), -np.inf]])
        for row, counts in enumerate(counted):
            with np.errstate(divide="ignore", invalid="ignore"):
                _, pairs, grad = topk_ce(ids, lp, x, [0], [row])
            q = np.exp(x[row] - x[row].max())
            q = q / q.sum()
            listed = -(np.exp(lp[0, :2]) * np.log(q[:2])).sum()
            if not counts:
                assert np.isclose(pairs[0], listed, rtol=1e-14) and (grad[row, 2:] == 0).all()
            elif row == 1:
                assert np.isclose(pairs[0], listed - short * np.log(q[2]), rtol=1e-13)
            else:
                assert pairs[0] > listed + 1e-6


@pytest.mark.parametrize("tail", [True, False])
def test_teacher_rows_that_held_nan(tail):
    nan = np.nan
    ids = np.array([[-1, -1], [-1, -1], [2, 0], [2, 0], [-1, 1]])
    lp = np.array([[nan, nan], [nan, -np.inf], [-0.5, nan], [-0.5, -1.5], [nan, -0.1]])
    x = np.linspace(-1, 1, 20).reshape(5, 4)
    _, pairs, grad = topk_ce(ids, lp, x, np.arange(5), np.arange(5), 1.0, tail)
    assert np.isnan(pairs).tolist() == [True, False, True, False, False]
    assert np.isnan(grad).all(1).tolist() == np.isnan(pairs).tolist() and pairs[1] == 0
