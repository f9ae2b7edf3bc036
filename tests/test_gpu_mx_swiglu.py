"""silu(gate) * up where a factor of it leaves float32's normal range and the product
does not: against the float64 oracle, as test_swiglu of test_gpu_mx.py.

The error is 2^-21 for gates from -80 up, as counted there (the exponential and the
reciprocal within 2^-23 each; 1 + e and three products rounded once each).  Below, e^-|g|
is taken as e^(128 - |g|) E E with E = e^-64: 128 - |g| is exact (|g| >= 64), the
exponential within 2^-23, each E rounded (2^-24), and four products rounded once each:
2^-23 + 2 * 2^-24 + 4 * 2^-24 = 2^-21 as well.
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
