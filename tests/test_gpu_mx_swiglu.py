"""silu(gate) * up where a factor of it leaves float32's normal range and the product
does not: against the float64 oracle, as test_swiglu of test_gpu_mx.py.

The error is at most 2^-21, as counted there, in units of 2^-23: e^-|g| = f 2^n has f from
the hardware's 2^x (1) of an argument below 1/2 with two roundings of 2^-26 (0.17), and
three products are rounded once each (1.5).  For g below zero the reciprocal of 1 + t and
its argument add 1 + 0.5 at most; where t is near 1 (the reciprocal near 1/2, where 1 ulp
is 1) half of f's error cancels in t / (1 + t): 0.59 + 1 + 0.25 + 1.5; where t vanishes
the reciprocal is near 1 (1 ulp is 0.5): 1.17 + 0.5 + 0.5 + 1.5 = 3.67, below 4.  2^n is
exact where the value is a normal number.
"""
import numpy as np
import pytest

from oracle import mx as O
from test_gpu_mx import TYPES, gen, matrix, near, values

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROWS, COLS = 32, 512

# ranges of the gates, the size of the ups: most products lie within float32's normal
# range.  Denormals in float32 only: bfloat16 has a few of them, whose products are
# multiples of one value, and so mostly lie on a border of the 4-bit values.
BOTH = ("f32", "bf16")
CASES = {
    "e^-|g| denormal or zero": ((-110.0, -88.0), 1e30, BOTH),
    "far past float32's exponential": ((-160.0, -110.0), 1e38, BOTH),
    "about the change of form": ((-82.0, -78.0), 1e10, BOTH),
    "denormal gates": ((-1e-40, 1e-40), 1e30, ("f32",)),
    "denormal ups": ((1e29, 1e30), 1e-40, ("f32",)),
    "small ups and factors": ((-20.0, -15.0), 1e-31, BOTH),
}


def check(gate, up):
    from paper_2505_14260_amd import mx
    ref = O.swiglu(gate.double().numpy(), up.double().numpy())
    q = matrix(*gate.shape)
    mx.swiglu(gate.cuda(), up.cuda(), q)
    near(values(q), ref, 2.0 ** -21)
    return ref


@pytest.mark.parametrize("name, type_", [(c, t) for c, v in CASES.items() for t in v[2]])
def test_factors_outside_the_normal_range(name, type_):
    (lo, hi), size, _ = CASES[name]
    g = gen(len(name))
    # in float64: the sizes are beyond float32's products
    gate = lo + (hi - lo) * torch.rand(ROWS, COLS, generator=g, dtype=torch.float64)
    up = size * (2 * torch.rand(ROWS, COLS, generator=g, dtype=torch.float64) - 1)
    gate, up = gate.float().to(TYPES[type_]), up.float().to(TYPES[type_])
    ref = check(gate, up)
    # most products do not vanish in 4 bits
    assert (np.abs(ref) > 2.0 ** -126).mean() > 0.5


def test_half_precision():
    """float16's largest ups bring e^-90 back into float32's normal range."""
    g = gen(5)
    gate = (-100 + 12 * torch.rand(ROWS, COLS, generator=g)).half()
    up = (60000 * (2 * torch.rand(ROWS, COLS, generator=g) - 1)).half()
    check(gate, up)


def test_one_far_gate_among_ordinary_ones():
    """A block's largest value may come from its only far gate."""
    g = gen(6)
    gate = torch.randn(ROWS, COLS, generator=g)
    up = torch.randn(ROWS, COLS, generator=g)
    gate[:, ::32], up[:, ::32] = -95.0, 1e38
    ref = check(gate, up)
    assert (np.abs(ref[:, ::32]) > 0.05).all()   # 95 e^-95 1e38 = 0.0525


def test_infinities_and_zeros():
    from paper_2505_14260_amd import mx
    inf, nan = float("inf"), float("nan")
    pairs = [(-inf, 1.0), (inf, 0.0), (nan, 1.0), (-90.0, nan), (-90.0, inf), (inf, 2.0),
             (-90.0, 0.0), (-1e30, 1e30), (0.0, 3e38), (-0.0, 1.0), (3e38, 0.0), (-200.0, -3e38)]
    gate, up = torch.zeros(1, 32 * len(pairs)), torch.zeros(1, 32 * len(pairs))
    for i, (a, b) in enumerate(pairs):
        gate[0, 32 * i], up[0, 32 * i] = a, b
    q = matrix(*gate.shape)
    mx.swiglu(gate.cuda(), up.cuda(), q)
    v = values(q).reshape(len(pairs), 32)
    # a NaN or an infinity makes its block NaN; the others are zero
    assert np.isnan(v[:6]).all() and (v[6:] == 0).all()


def test_overflow_before_the_exponential():
    """|g u| past float32's largest value, |silu(g) u| below it."""
    g = gen(7)
    gate = -40 * torch.rand(ROWS, COLS, generator=g)
    up = 3e38 * (2 * torch.rand(ROWS, COLS, generator=g) - 1)
    ref = check(gate, up)
    assert np.abs(ref).max() < 3e38
    assert ((gate.double() * up.double()).abs() > 3.5e38).double().mean() > 0.5
