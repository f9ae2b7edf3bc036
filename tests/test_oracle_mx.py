"""The 4-bit format's oracle against worked values and the format's bounds."""
import numpy as np
import pytest

from oracle import mx

PI = [3.14159, -1.0, 0.2, 0.1]


def block(vals):
    x = np.zeros((1, 32))
    x[0, :len(vals)] = vals
    return x


def test_worked_block():
    # largest 3.14: s = 2^(1 - 2) = 1/2; x / s = 6.28, -2, 0.4, 0.2 -> 6, -2, 0.5, 0
    assert list(mx.term(block(PI))[0, :4]) == [3.0, -1.0, 0.25, 0.0]
    # what is left: 0.14159, 0, -0.05, 0.1; s = 2^(-3 - 2); 4.53, 0, -1.6, 3.2 -> 4, 0, -1.5, 3
    left = block(PI) - mx.term(block(PI))
    assert list(mx.term(left)[0, :4]) == [4 / 32, 0.0, -1.5 / 32, 3 / 32]


def test_ties_go_to_the_even_code():
    ties = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    want = [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0]
    got = mx.term(block([4.0] + ties + [-t for t in ties]))[0]
    assert list(got[1:8]) == want and list(got[8:15]) == [-w for w in want]


def test_saturation_scale_range_and_special_blocks():
    assert mx.term(block([7.9]))[0, 0] == 6.0      # 7.9 lies under 8 = 2^3: s = 1
    assert mx.term(block([8.0]))[0, 0] == 8.0
    assert mx.term(block([2.0 ** -149]))[0, 0] == 0.0   # s is 2^-127 at least
    assert mx.term(block([2.0 ** -127]))[0, 0] == 2.0 ** -127
    assert mx.term(block([3.0e38]))[0, 0] == 6 * 2.0 ** 125
    assert not mx.term(block([0.0])).any()
    x = np.ones((1, 64))
    x[0, 40] = np.inf
    v = mx.term(x)
    assert (v[0, :32] == 1).all() and np.isnan(v[0, 32:]).all()


@pytest.mark.parametrize("cols", [1, 31, 32, 33, 100])
def test_error_bounds_and_idempotence(cols):
    x = np.random.default_rng(cols).standard_normal((50, cols)) * 10.0 ** np.arange(-5, 5).repeat(5)[:, None]
    hi = mx.term(x)
    pad = np.zeros((50, -(-cols // 32) * 32))
    pad[:, :cols] = np.abs(x)
    top = pad.reshape(50, -1, 32).max(-1).repeat(32, 1)[:, :cols]
    # half the widest step, 1 s, or the saturation's 2 s, with s <= top / 4
    assert (np.abs(x - hi) <= top / 2).all()
    assert (np.abs(x - mx.quantised(x, 2)) <= top / 8).all()
    assert (mx.term(hi) == hi).all()


def test_norm_and_swiglu_against_direct_forms():
    rng = np.random.default_rng(3)
    s, g = rng.standard_normal((4, 7)), rng.standard_normal(7)
    v = mx.rms_norm(s, np.ones(7), 0.0)
    assert np.allclose((v * v).mean(-1), 1, rtol=0, atol=1e-14)
    assert np.allclose(mx.rms_norm(s, g, 0.0), v * g, rtol=1e-14)
    gate = np.linspace(-30, 30, 61)[None]
    assert np.allclose(mx.swiglu(gate, np.ones_like(gate)), gate / (1 + np.exp(-gate)), rtol=1e-13)
    assert mx.swiglu(np.array([[-800.0, 800.0]]), np.ones((1, 2))).tolist() == [[0.0, 800.0]]
