"""Products on every kernel that the plan may pick (tests/test_mx_plan.py shows on the
CPU that PRODUCTS reaches them all), compared over the whole output, in all three types.

Tolerances: as for test_product of test_gpu_mx.py (float32 sums of n = k * terms
products: n 2^-24 of the sum of |x w|, half a step of the output's type; sums whose
every partial sum float32 holds are exact).  The reference is in float64 on the GPU;
its quantisation is compared with oracle/mx.py on some of the rows.
"""
import numpy as np
import pytest

from oracle import mx as O
from test_gpu_mx import HALF_STEP, TYPES, gen, matrix

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# (columns n, length k): rows.  None of n is a multiple of 16, none of k of 128.
PRODUCTS = {
    (515, 1500): (10, 20, 60),
    (515, 4700): (10, 31, 100, 500),
    (1777, 7700): (300, 500),
    (4611, 2100): (1, 10, 16, 20, 33, 63, 65, 129),
    (4611, 4700): (10, 17, 40, 63),
    (8637, 2900): (10, 20, 31, 40, 63),
    (13291, 4700): (5, 16, 20, 31, 40, 129, 500, 1000),
    (32001, 4200): (10, 16, 20, 31, 60, 200, 500, 641),
    (35003, 1100): (17, 1000),
    (52003, 300): (1, 17, 500),
}


def power(e):
    """2^e in float64, from its bits (torch's ldexp takes a rounded pow)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def term(x):
    """oracle/mx.py's term of finite float64 values, on the GPU."""
    rows, cols = x.shape
    b = torch.zeros(rows, -(-cols // 32) * 32, dtype=torch.float64, device=x.device)
    b[:, :cols] = x
    b = b.view(rows, -1, 32)
    top = b.abs().amax(-1, keepdim=True)
    e = torch.where(top > 0, torch.frexp(top)[1] - 3, -127).clamp(-127, 127)
    scale = power(e)
    a = b.abs() / scale
    grid = torch.from_numpy(O.GRID).to(x.device)
    code = torch.zeros_like(a, dtype=torch.int64)
    for i in range(7):
        mid = (grid[i] + grid[i + 1]) / 2
        code += (a >= mid) if i % 2 else (a > mid)
    v = (torch.copysign(grid[code], b) * scale).view(rows, -1)[:, :cols].contiguous()
    some = [0, rows // 2, rows - 1]
    assert np.array_equal(v[some].cpu().numpy(), O.term(x[some].cpu().numpy()))
    return v


def last_bit(v):
    """Per row, the largest power of two that divides all of its values."""
    m, e = torch.frexp(v)
    i = (m.abs() * 2.0 ** 53).to(torch.int64)
    low = (i & -i).double() * power(e - 53)
    return torch.where(v != 0, low, torch.inf).amin(1)


@pytest.mark.parametrize("terms", [1, 2])
@pytest.mark.parametrize("n, k", list(PRODUCTS), ids=lambda v: str(v))
def test_every_kernel(n, k, terms):
    from paper_2505_14260_amd import mx
    rows = PRODUCTS[n, k]
    x = torch.randn(max(rows), k, generator=gen(n)).cuda()
    w = (0.02 * torch.randn(n, k, generator=gen(k))).bfloat16().cuda()
    qw = mx.quantize(w, matrix(n, k, "weight", 1))
    xv, wv = term(x.double()), term(w.double())
    if terms == 2:
        xv = xv + term(x.double() - xv)
    wt = wv.t().contiguous()
    full, size = xv @ wt, xv.abs() @ wt.abs()
    firm = size < 2.0 ** 24 * torch.outer(last_bit(xv), last_bit(wv))
    for r in rows:
        qx = mx.quantize(x[:r], matrix(r, k, "rows", terms))
        for type_, pad, offset in (("f32", 0, 0), ("f32", 3, 1), ("bf16", 5, 4), ("f16", 1, 0)):
            print(f"case: {r} x {n} x {k}, {terms} terms, {type_}, pad {pad}", flush=True)
            buf = torch.full((offset + (r + 2) * (n + pad),), -3.0, dtype=TYPES[type_], device="cuda")
            out = buf[offset:].view(r + 2, n + pad)
            mx.product(qx, qw, out[:r, :n])
            got, ref = out[:r, :n].double(), full[:r]
            assert (buf[:offset] == -3).all() and (out[:, n:] == -3).all() and (out[r:] == -3).all()
            if type_ == "f32":
                assert firm[:r].double().mean() > 0.5 and (got == ref)[firm[:r]].all()
            tiny = 2.0 ** -25 if type_ == "f16" else 0.0   # half a step of its denormals
            bound = k * terms * 2.0 ** -24 * size[:r] * (1 + HALF_STEP[type_]) \
                + HALF_STEP[type_] * ref.abs() + tiny
            assert (got - ref).abs().le(bound).all()
            # far inside the bound above: a tile gone wrong moves the result by 2^-8 and more
            assert float((got - ref).norm()) <= (2.0 ** -12 + HALF_STEP[type_]) * float(ref.norm())
