"""The oracle of the operators on logits, pinned by hand-made rows and closed forms (CPU)."""
import numpy as np
import pytest

from oracle import logits as O


def test_order_and_log_sum_exp():
    row = np.array([1.0, np.nan, 3.0, -0.0, 0.0, 3.0, -np.inf])
    v, i, lse = O.top(row, 7)
    assert i.tolist() == [2, 5, 0, 3, 4, 1, 6]
    assert v.tolist() == [3, 3, 1, 0, 0, -np.inf, -np.inf]
    assert abs(lse - np.log(2 * np.e ** 3 + np.e + 2)) < 1e-15
    assert O.top(np.full(3, -np.inf), 2)[2] == -np.inf and O.top(np.array([np.inf, 1]), 1)[2] == np.inf


def test_what_stays():
    p = np.array([0.1, 0.4, 0.05, 0.3, 0.15])
    row = np.log(p)
    def ids(**how):
        return O.stay(row, **how)[0].tolist()
    assert ids() == [1, 3, 4, 0, 2] and ids(top_k=2) == [1, 3] and ids(temperature=0.0) == [1]
    assert ids(top_p=0.69) == [1, 3] and ids(top_p=0.71) == [1, 3, 4] and ids(top_p=1e-9) == [1]
    assert ids(min_p=0.3) == [1, 3, 4] and ids(min_p=1.0) == [1]
    # top-p counts the mass of what top-k left: 0.4 of 0.7 is 0.57
    assert ids(top_k=2, top_p=0.57) == [1] and ids(top_k=2, top_p=0.58) == [1, 3]
    # a temperature of 1/2 squares the weights: 0.16 of 0.285
    assert ids(temperature=0.5, top_p=0.56) == [1] and ids(temperature=0.5, top_p=0.57) == [1, 3]
    assert len(O.stay(np.full(4, np.nan))[0]) == 0


@pytest.mark.parametrize("u, want", [(0.0, 0), (0.0999, 0), (0.1001, 1), (0.4999, 1), (0.5001, 2),
                                     (0.5499, 2), (0.5501, 3), (0.8501, 4), (1.0, 4), (-1.0, 0),
                                     (float("nan"), 0)])
def test_inverse_sampling(u, want):
    row = np.log([0.1, 0.4, 0.05, 0.3, 0.15])
    token, lp, _ = O.sample(row, u)
    assert token == want and abs(lp - row[want]) < 1e-12
    # among ids 1 and 3 alone
    token, lp, _ = O.sample(row, u, top_k=2)
    assert token == (1 if not u > 4 / 7 else 3)
    assert O.sample(np.full(3, -np.inf), u)[:2] == (-1, -np.inf)


def test_divergence_and_gradient():
    rng = np.random.default_rng(0)
    x = rng.normal(size=30)
    # all entries at T = 1: the Kullback-Leibler divergence; none with itself
    t = rng.normal(size=30)
    loss, lse, dx, p, q = O.distill(x, np.arange(30), t, 1.0)
    qq, pp = np.exp(t) / np.exp(t).sum(), np.exp(x) / np.exp(x).sum()
    assert abs(loss - (qq * np.log(qq / pp)).sum()) < 1e-14 and np.allclose(dx, pp - qq, atol=1e-15)
    assert abs(O.distill(x, np.arange(30), x + 3, 1.0)[0]) < 1e-14
    # one entry: the cross-entropy of a label
    loss, lse, dx, _, _ = O.distill(x, [7], [123.0], 1.0)
    assert abs(loss - (lse - x[7])) < 1e-14
    # entries out of range are none, one that comes twice counts twice
    a = O.distill(x, [3, 9, -1, 30], [1.0, 2.0, 9.0, 9.0], 2.0)
    b = O.distill(x, [3, 9], [1.0, 2.0], 2.0)
    assert a[0] == b[0] and np.array_equal(a[2], b[2])
    c = O.distill(x, [3, 9, 9], [1.0, 2.0, 2.0], 2.0)
    w = np.exp([0.5, 1.0, 1.0]) / np.exp([0.5, 1.0, 1.0]).sum()
    assert abs(c[4][9] - 2 * w[1]) < 1e-15
    h, T = 1e-5, 2.0
    for k in (0, 3, 9):
        d = x.copy()
        d[k] += h
        e = x.copy()
        e[k] -= h
        num = (O.distill(d, [3, 9, 9], [1.0, 2.0, 2.0], T)[0]
               - O.distill(e, [3, 9, 9], [1.0, 2.0, 2.0], T)[0]) / (2 * h)
        assert abs(num - c[2][k]) < 1e-9
