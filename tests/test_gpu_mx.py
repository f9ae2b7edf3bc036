"""The microscaled operators on the GPU against the float64 oracle (oracle/mx.py).

Quantisation is exact: the same values as the oracle's, bit for bit.  The norm and
SwiGLU round what they computed in float32 or better to 4 bits, which moves by a
whole step where it lies next to a border: a block must equal the oracle's unless
the oracle's own block changes when its input moves by the operator's error, DELTA
(relative), either way.
  norm: the sum of x and y is the same float32 sum on both sides; float64, then one
  rounding to float32 (2^-24): 2^-23.
  swiglu: e^-|g| within 2^-23 and the reciprocal within 2^-23, the sum 1 + e and up to
  three products rounded once each (2^-24): 2 * 2^-23 + 4 * 2^-24 = 2^-21.
Products: float32 sums of n = cols * terms products: at most n 2^-24 of the sum of
|x w| (each sum rounded at no more than that size), plus half a step of the output
type relative to the value.  Where all products are multiples of a u with the sum of
|x w| below 2^24 u, float32 holds every partial sum in any order: those sums must be
exact.  Inputs of one scale have mostly such sums (a block's last bits lie 5 below
its largest value's; a block of one value, as of 129 columns, may lie anywhere).
"""
import numpy as np
import pytest

from oracle import mx as O

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def wild(rows, cols, seed, spread=8):
    """Rows of very different sizes, blocks too, with exact zeros and ties."""
    g = gen(seed)
    x = torch.randn(rows, cols, generator=g)
    x = x * torch.exp2(torch.randint(-spread, spread + 1, (rows, 1), generator=g).float())
    x = x * torch.exp2(torch.randint(-3, 4, (1, -(-cols // 32)), generator=g).float()
                       .repeat_interleave(32, 1)[:, :cols])
    pick = torch.rand(rows, cols, generator=g)
    x = torch.where(pick < 0.05, 0.0, x)
    return torch.where(pick > 0.9, torch.round(x * 4) / 4, x)


def strided(x, pad, offset=0):
    """x on the GPU in rows `pad` values wider, `offset` values past the start."""
    rows, cols = x.shape
    buf = torch.full((rows * (cols + pad) + offset,), 7.0, dtype=x.dtype, device="cuda")
    v = buf[offset:].view(rows, cols + pad)[:, :cols]
    v.copy_(x)
    return v


def matrix(rows, cols, layout="rows", terms=2):
    """A quantised matrix whose buffers hold nothing useful yet."""
    from paper_2505_14260_amd import mx
    q = mx.MX(rows, cols, layout=layout, terms=terms)
    q.codes.fill_(0xF7)
    q.scales.fill_(0xF1)
    return q


def values(q):
    from paper_2505_14260_amd import mx
    return mx.dequantize(q, torch.empty(q.shape, device="cuda")).double().cpu().numpy()


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


SIZES = [(1, 1), (1, 31), (2, 32), (3, 33), (15, 127), (16, 128), (17, 129), (5, 511), (4, 512),
         (33, 513), (2, 1000), (70, 2056), (1, 18944)]


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("layout, terms", [("rows", 1), ("rows", 2), ("weight", 1)])
def test_quantise_is_exact(layout, terms, type_):
    from paper_2505_14260_amd import mx
    for i, (rows, cols) in enumerate(SIZES):
        print(f"case: {rows} x {cols}", flush=True)
        x = wild(rows, cols, i, 4 if type_ == "f16" else 8).to(TYPES[type_])
        want = O.quantised(x.double().numpy(), terms)
        for pad, offset in ((0, 0), (8, 8), (3, 1)):
            q = matrix(rows, cols, layout, terms)
            mx.quantize(strided(x, pad, offset), q)
            assert same(values(q), want.astype(np.float32).astype(np.float64)), (rows, cols, pad)


@pytest.mark.parametrize("layout, terms", [("rows", 1), ("rows", 2), ("weight", 1)])
def test_quantise_special_values(layout, terms):
    from paper_2505_14260_amd import mx
    x = torch.randn(20, 200, generator=gen(1))
    x[0] = 0
    x[1, 5], x[1, 64], x[2, 199], x[3, 100] = float("nan"), float("inf"), float("-inf"), -0.0
    x[4] *= 2.0 ** -130          # denormal, below the smallest scale
    x[5] *= 2.0 ** 120
    x[6, :32] = torch.finfo(torch.float32).max
    x[7] = 2.0 ** -149
    x[8, :16] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 4.0] * 2)
    q = matrix(20, 200, layout, terms)
    mx.quantize(x.cuda(), q)
    want = O.quantised(x.double().numpy(), terms).astype(np.float32).astype(np.float64)
    assert same(values(q), want)
    assert np.isnan(want[1, :32]).all() and np.isnan(want[1, 64:96]).all()
    assert np.isfinite(want[1, 32:64]).all() and np.isnan(want[2, 192:]).all()


@pytest.mark.parametrize("type_", list(TYPES))
def test_dequantise_types_strides_and_what_lies_beside(type_):
    from paper_2505_14260_amd import mx
    x = wild(9, 77, 5, 3)
    q = matrix(9, 77)
    mx.quantize(x.cuda(), q)
    want = torch.from_numpy(O.quantised(x.double().numpy(), 2)).to(TYPES[type_])
    for pad, offset in ((0, 0), (3, 8), (11, 1)):
        buf = torch.full((offset + 12 * (77 + pad),), -3.0, dtype=TYPES[type_], device="cuda")
        out = buf[offset:].view(12, 77 + pad)
        mx.dequantize(q, out[:9, :77])
        assert torch.equal(out[:9, :77].cpu(), want)
        assert (buf[:offset] == -3).all() and (out[:, 77:] == -3).all() and (out[9:] == -3).all()


def near(got, ref, delta):
    """got must be the oracle's quantised ref, block by block, where the oracle's
    block stays the same under a relative change of delta."""
    a, lo, hi = (O.quantised(ref * f, 2) for f in (1.0, 1 - delta, 1 + delta))
    firm = O.block_same(a, lo) & O.block_same(a, hi)
    # the oracle's unmoved blocks are scaled by 1 -+ delta only through their values
    ok = O.block_same(got, a.astype(np.float32).astype(np.float64))
    assert (ok | ~firm).all(), np.argwhere(firm & ~ok)[:5]
    # a value is next to one of some 30 borders a binade with chance 2^6 delta
    assert (~firm).mean() <= 0.01 + 32 * 2.0 ** 7 * delta
    top = np.abs(np.pad(ref, ((0, 0), (0, -ref.shape[1] % 32)))).reshape(len(ref), -1, 32).max(-1)
    far = np.abs(np.pad(got - ref, ((0, 0), (0, -ref.shape[1] % 32)))).reshape(len(ref), -1, 32).max(-1)
    # top / 8 holds where s <= top / 4; where s is held up at 2^-127 (top < 2^-125),
    # what is below half the smallest step, 2^-128, is lost: 2^-129 at most
    assert (far <= top / 8 * (1 + 2.0 ** -10) + 2.0 ** -129).all()


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("rows, cols", [(1, 1), (3, 8), (2, 33), (5, 512), (4, 2040), (3, 2049),
                                        (7, 3584), (2, 4097), (70, 4096), (2, 8191), (1, 8192)])
def test_norm(rows, cols, type_):
    from paper_2505_14260_amd import mx
    t = TYPES[type_]
    x = (wild(rows, cols, rows + cols, 3)).to(t)
    y = torch.randn(rows, cols, generator=gen(7)).to(t)
    gain = (1 + 0.2 * torch.randn(cols, generator=gen(8))).bfloat16()
    for use_y, pad, offset in ((True, 0, 0), (False, 8, 8), (True, 5, 1)):
        print(f"case: y {use_y}, pad {pad}", flush=True)
        s = x.float() + y.float() if use_y else x.float()
        ref = O.rms_norm(s.double().numpy(), gain.double().numpy(), np.float64(np.float32(1e-5)))
        xd, yd = strided(x, pad, offset), strided(y, pad, offset) if use_y else None
        out = strided(torch.zeros_like(x), pad, offset)
        q = matrix(rows, cols)
        mx.resid_norm(xd, yd, gain.cuda(), 1e-5, out, q)
        assert torch.equal(out.cpu(), s.to(t))
        near(values(q), ref, 2.0 ** -23)
        # in place, and without the sum
        for target in (xd, yd, None):
            if target is None and not use_y:
                continue
            q2 = matrix(rows, cols)
            xs, ys = xd.clone(), yd.clone() if use_y else None
            to = xs if target is xd else ys if target is not None else None
            mx.resid_norm(xs, ys, gain.cuda(), 1e-5, to, q2)
            assert torch.equal(q.codes, q2.codes) and torch.equal(q.scales, q2.scales)
            if to is not None:
                assert torch.equal(to.cpu(), s.to(t))


def test_norm_special_rows():
    from paper_2505_14260_amd import mx
    x = torch.randn(6, 96, generator=gen(2))
    x[0] = 0
    x[1, 40] = float("nan")
    x[2, 40] = float("inf")
    x[3] *= 1e18                       # squares past float32
    x[4] *= 1e-25                      # squares below it
    gain = torch.ones(96, dtype=torch.bfloat16)
    q = matrix(6, 96)
    mx.resid_norm(x.cuda(), None, gain.cuda(), 0.0, None, q)
    v = values(q)
    assert np.isnan(v[:2]).all()       # 0 / 0, and a NaN in the mean
    assert np.isnan(v[2, 32:64]).all() and (v[2, :32] == 0).all()   # inf / inf; 1 / inf
    near(v[3:], O.rms_norm(x[3:].double().numpy(), np.ones(96), 0.0), 2.0 ** -23)
    mx.resid_norm(x.cuda(), None, gain.cuda(), 1e-6, None, q)
    assert (values(q)[0] == 0).all()


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("rows, cols", [(1, 1), (3, 33), (4, 688), (17, 2880), (2, 11008), (1, 18944)])
def test_swiglu(rows, cols, type_):
    from paper_2505_14260_amd import mx
    t = TYPES[type_]
    both = (3 * torch.randn(rows, 2 * cols, generator=gen(cols))).to(t)
    both[0, 0] = -100.0
    ref = O.swiglu(both[:, :cols].double().numpy(), both[:, cols:].double().numpy())
    for pad, offset in ((0, 0), (3, 1)):
        b = strided(both, pad, offset)
        q = matrix(rows, cols)
        mx.swiglu(b[:, :cols], b[:, cols:], q)
        near(values(q), ref, 2.0 ** -21)


def operands(rows, n, k, terms, seed, gentle):
    x = torch.randn(rows, k, generator=gen(seed)) if gentle else wild(rows, k, seed)
    w = torch.randn(n, k, generator=gen(seed + 1)) * 0.02 if gentle else wild(n, k, seed + 1)
    from paper_2505_14260_amd import mx
    qx, qw = matrix(rows, k, "rows", terms), matrix(n, k, "weight", 1)
    mx.quantize(x.cuda(), qx)
    mx.quantize(w.bfloat16().cuda(), qw)
    return qx, qw, O.quantised(x.double().numpy(), terms), O.term(w.bfloat16().double().numpy())


def last_bit(v):
    """Per row, the largest power of two that divides all of its values."""
    m, e = np.frexp(v)
    i = np.abs(m * 2.0 ** 53).astype(np.int64)
    low = np.ldexp((i & -i).astype(np.float64), e - 53)
    return np.where(v != 0, low, np.inf).min(1)


# both sides of every tile of 16 rows or columns, of 128 columns of K and of the
# groups of 512, and of the row counts at which another kernel takes over
ROWS = [1, 2, 15, 16, 17, 31, 33, 48, 63, 64, 65, 100, 127, 128, 129, 200, 255, 257]
NK = [(1, 1), (3, 31), (16, 32), (17, 33), (64, 127), (100, 128), (257, 129), (130, 511), (128, 512),
      (48, 513), (515, 1000), (256, 4096), (96, 4100), (272, 11008)]


@pytest.mark.parametrize("terms", [1, 2])
@pytest.mark.parametrize("gentle", [True, False], ids=["gentle", "wild"])
def test_product(gentle, terms):
    from paper_2505_14260_amd import mx
    for i, (n, k) in enumerate(NK):
        rows = ROWS if i % 3 == 0 else ROWS[i % 4::4]
        qx, qw, x, w = operands(max(rows), n, k, terms, i, gentle)
        full, size = x @ w.T, np.abs(x) @ np.abs(w).T
        with np.errstate(invalid="ignore", over="ignore"):
            firm = size < 2.0 ** 24 * np.outer(last_bit(x), last_bit(w))
        for r in rows:
            type_ = ("f32", "bf16", "f16")[(r + i) % 3] if not gentle else "f32"
            pad, offset = ((0, 0), (4, 4), (3, 1))[(r + i) % 3]
            print(f"case: {r} x {n} x {k}, {type_}, pad {pad}", flush=True)
            part = matrix(r, k, "rows", terms)
            part.codes.copy_(qx.codes[:part.codes.numel()])
            part.scales.copy_(qx.scales[:part.scales.numel()])
            buf = torch.full((offset + (r + 2) * (n + pad),), -3.0, dtype=TYPES[type_], device="cuda")
            out = buf[offset:].view(r + 2, n + pad)
            mx.product(part, qw, out[:r, :n])
            got = out[:r, :n].double().cpu().numpy()
            assert (buf[:offset] == -3).all() and (out[:, n:] == -3).all() and (out[r:] == -3).all()
            if type_ == "f32":
                off = firm[:r] & (got != full[:r])
                assert not off.any(), np.argwhere(off)[:5]
                assert not gentle or firm.mean() > 0.5
            if type_ == "f16":     # past 65504 the type has no value
                fine = np.abs(full[:r]) < 60000
            else:
                fine = np.ones_like(full[:r], dtype=bool)
            tiny = 2.0 ** -25 if type_ == "f16" else 0.0   # half a step of its denormals
            bound = k * terms * 2.0 ** -24 * size[:r] * (1 + HALF_STEP[type_]) \
                + HALF_STEP[type_] * np.abs(full[:r]) + tiny
            assert (np.abs(got - full[:r]) <= bound)[fine].all()


@pytest.mark.parametrize("rows, n, k", [
    (635, 22003, 4100),    # workgroup tiles of 128 x 256
    (1030, 12289, 4096), (2050, 4100, 11000),
    (3121, 4090, 11000),   # of 256 x 256
    (385, 32001, 4096)])
@pytest.mark.parametrize("terms, type_", [(2, "f32"), (1, "bf16"), (2, "f16")])
def test_product_of_many_rows(rows, n, k, terms, type_):
    """The largest workgroup tiles, cut at their last rows and columns (the reference:
    the oracle's values, multiplied in float64 on the GPU)."""
    from paper_2505_14260_amd import mx
    g = gen(rows)
    x, w = torch.randn(rows, k, generator=g), (torch.randn(n, k, generator=g) * 0.02).bfloat16()
    qx, qw = matrix(rows, k, "rows", terms), matrix(n, k, "weight", 1)
    mx.quantize(x.cuda(), qx)
    mx.quantize(w.cuda(), qw)
    buf = torch.full((rows + 1, n + 3), -3.0, dtype=TYPES[type_], device="cuda")
    mx.product(qx, qw, buf[:rows, :n])
    assert (buf[rows:] == -3).all() and (buf[:, n:] == -3).all()
    a, b = O.quantised(x.double().numpy(), terms), O.term(w.double().numpy())
    u = torch.outer(*(torch.from_numpy(last_bit(v)).cuda() for v in (a, b)))
    a, b = torch.from_numpy(a).cuda(), torch.from_numpy(b).cuda()
    full, size = a @ b.t().contiguous(), a.abs() @ b.abs().t().contiguous()
    got = buf[:rows, :n].double()
    if type_ == "f32":
        firm = size < 2.0 ** 24 * u
        assert firm.double().mean() > 0.5 and (got == full)[firm].all()
    bound = k * terms * 2.0 ** -24 * size * (1 + HALF_STEP[type_]) + HALF_STEP[type_] * full.abs() \
        + (2.0 ** -25 if type_ == "f16" else 0.0)
    assert (got - full).abs().le(bound).all()
    # far inside the bound above: a tile gone wrong moves the result by 2^-8 and more
    assert float((got - full).norm()) <= (2.0 ** -12 + HALF_STEP[type_]) * float(full.norm())


@pytest.mark.parametrize("rows", [3, 40, 130, 300])
def test_product_with_nan_blocks_and_zeros(rows):
    """A NaN block of x takes its row, one of w its column; the rest is as ever."""
    from paper_2505_14260_amd import mx
    x, w = torch.randn(rows, 300, generator=gen(1)), torch.randn(80, 300, generator=gen(2))
    x[2, 7], w[33, 290] = float("nan"), float("inf")
    x[0], w[5] = 0, 0
    qx, qw = matrix(rows, 300), matrix(80, 300, "weight", 1)
    mx.quantize(x.cuda(), qx)
    mx.quantize(w.cuda(), qw)
    out = mx.product(qx, qw, torch.empty(rows, 80, device="cuda")).double().cpu().numpy()
    ref = O.quantised(x.double().numpy(), 2) @ O.term(w.double().numpy()).T
    assert np.isnan(out[2]).all() and np.isnan(out[:, 33]).all()
    assert same(out, ref)


def test_offsets_past_32_bits():
    """A weight of 8.6e9 values (17 GB of bfloat16, 4.9 GB of codes), its last rows
    against the oracle, with products of few and of many rows."""
    from paper_2505_14260_amd import mx
    rows, cols = 131_073, 65_544
    w = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    for r in range(0, rows, 16384):
        w[r:r + 16384].normal_()
    q = matrix(rows, cols, "weight", 1)
    assert q.codes.numel() > 2 ** 32
    print("case: quantise", flush=True)
    mx.quantize(w, q)
    tail = O.term(w[-40:].double().cpu().numpy())
    print("case: values", flush=True)
    out = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    mx.dequantize(q, out)
    assert same(out[-40:].double().cpu().numpy(), tail)
    del out, w
    for m in (3, 300):
        print(f"case: {m} rows", flush=True)
        x = torch.randn(m, cols, generator=gen(m))
        qx = matrix(m, cols)
        mx.quantize(x.cuda(), qx)
        y = torch.empty(m, rows, device="cuda")
        mx.product(qx, q, y)
        v = O.quantised(x.double().numpy(), 2)
        full, size = v @ tail.T, np.abs(v) @ np.abs(tail).T
        got = y[:, -40:].double().cpu().numpy()
        assert (np.abs(got - full) <= 2 * cols * 2.0 ** -24 * size).all()
        # a relative error of 2^-10 of the sums' own size would be a tile gone wrong
        assert np.linalg.norm(got - full) <= 2.0 ** -10 * np.linalg.norm(full)


@pytest.mark.parametrize("rows", [127, 128, 129, 256, 271, 1000])
def test_norm_of_many_rows(rows):
    """From 128 rows on they run in another order; a row's result does not depend on
    how many there are."""
    from paper_2505_14260_amd import mx
    x, y = wild(rows, 1100, rows, 3), torch.randn(rows, 1100, generator=gen(9))
    gain = (1 + 0.2 * torch.randn(1100, generator=gen(8))).bfloat16()
    xd, yd, gd = x.cuda(), y.cuda(), gain.cuda()
    out, q = torch.full((rows + 3, 1100), -3.0, device="cuda"), matrix(rows, 1100)
    mx.resid_norm(xd, yd, gd, 1e-5, out[:rows], q)
    assert torch.equal(out[:rows].cpu(), x + y) and (out[rows:] == -3).all()
    v = values(q)
    near(v, O.rms_norm((x + y).double().numpy(), gain.double().numpy(),
                       np.float64(np.float32(1e-5))), 2.0 ** -23)
    for r in range(0, rows, 50):
        n = min(50, rows - r)
        part = matrix(n, 1100)
        mx.resid_norm(xd[r:r + n], yd[r:r + n], gd, 1e-5, None, part)
        assert same(values(part), v[r:r + n])


@pytest.mark.parametrize("layout", ["rows", "weight"])
@pytest.mark.parametrize("type_", ["f32", "f16"])
def test_values_of_a_large_matrix(layout, type_):
    """One term of many rows, whose last are no multiple of four or sixteen."""
    from paper_2505_14260_amd import mx
    x = wild(4101, 4100, 3, 3).to(TYPES[type_])
    q = matrix(4101, 4100, layout, 1)
    mx.quantize(x.cuda(), q)
    out = torch.full((4102, 4103), -3.0, dtype=TYPES[type_], device="cuda")
    mx.dequantize(q, out[:4101, :4100])
    assert torch.equal(out[:4101, :4100].cpu(), torch.from_numpy(O.term(x.double().numpy())).to(TYPES[type_]))
    assert (out[4101:] == -3).all() and (out[:, 4100:] == -3).all()


def test_most_rows():
    """2^23 rows of few columns: the operators' largest grids."""
    from paper_2505_14260_amd import mx
    rows, cols = 1 << 23, 3
    x = torch.randn(rows, cols, device="cuda")
    y = torch.randn(rows, cols, device="cuda")
    gain = torch.ones(cols, dtype=torch.bfloat16, device="cuda")
    pick = torch.tensor([0, 1, 15, 16, 127, 128, 1 << 20, 5_000_001, rows - 17, rows - 1])
    a, b = (t[pick.cuda()].cpu() for t in (x, y))
    q, out = matrix(rows, cols), torch.empty(rows, cols, device="cuda")

    def got():
        return mx.dequantize(q, out)[pick.cuda()].double().cpu().numpy()
    print("case: quantise", flush=True)
    mx.quantize(x, q)
    assert same(got(), O.quantised(a.double().numpy(), 2))
    print("case: norm", flush=True)
    mx.resid_norm(x, y, gain, 1e-5, None, q)
    ref = O.rms_norm((a + b).double().numpy(), np.ones(cols), np.float64(np.float32(1e-5)))
    near(got(), ref, 2.0 ** -23)
    print("case: swiglu", flush=True)
    mx.swiglu(x, y, q)
    near(got(), O.swiglu(a.double().numpy(), b.double().numpy()), 2.0 ** -21)
    print("case: product", flush=True)
    w = torch.randn(5, cols, generator=gen(1))
    qw = mx.quantize(w.cuda(), matrix(5, cols, "weight", 1))
    mx.quantize(x, q)
    y = mx.product(q, qw, torch.empty(rows, 5, device="cuda"))[pick.cuda()].double().cpu().numpy()
    v, u = O.quantised(a.double().numpy(), 2), O.term(w.double().numpy())
    assert (np.abs(y - v @ u.T) <= 2 * cols * 2.0 ** -24 * (np.abs(v) @ np.abs(u).T)).all()


def test_longest_rows():
    """2^20 columns."""
    from paper_2505_14260_amd import mx
    cols = 1 << 20
    w = torch.randn(33, cols, generator=gen(1)).bfloat16()
    qw = mx.quantize(w.cuda(), matrix(33, cols, "weight", 1))
    u = O.term(w.double().numpy())
    assert same(values(qw), u)
    for m in (5, 70):
        print(f"case: {m} rows", flush=True)
        x = torch.randn(m, cols, generator=gen(m))
        qx = mx.quantize(x.cuda(), matrix(m, cols))
        v = O.quantised(x.double().numpy(), 2)
        assert same(values(qx), v)
        got = mx.product(qx, qw, torch.empty(m, 33, device="cuda")).double().cpu().numpy()
        full, size = v @ u.T, np.abs(v) @ np.abs(u).T
        assert (np.abs(got - full) <= 2 * cols * 2.0 ** -24 * size).all()
        # a relative error of 2^-10 of the sums' own size would be a tile gone wrong
        assert np.linalg.norm(got - full) <= 2.0 ** -10 * np.linalg.norm(full)


def test_empty_matrices():
    from paper_2505_14260_amd import mx
    q, w = mx.MX(0, 64), mx.MX(16, 64, layout="weight")
    e = torch.empty(0, 64, device="cuda")
    mx.quantize(e, q)
    mx.dequantize(q, e)
    mx.resid_norm(e, e, torch.ones(64, dtype=torch.bfloat16, device="cuda"), 1e-5, e, q)
    mx.swiglu(e, e, q)
    mx.product(q, w, torch.empty(0, 16, device="cuda"))
    mx.product(mx.MX(4, 64), mx.MX(0, 64, layout="weight"), torch.empty(4, 0, device="cuda"))
    torch.cuda.synchronize()


def ffn(x, y, gain, wgu, wd, bufs):
    """One decoder FFN in 4 bits, as a program would run it."""
    from paper_2505_14260_amd import mx
    s, q, gu, act, out = bufs
    F = act.shape[1]
    mx.resid_norm(x, y, gain, 1e-5, s, q)
    mx.product(q, wgu, gu)
    mx.swiglu(gu[:, :F], gu[:, F:], act)
    return mx.product(act, wd, out)


def ffn_setup(rows, d, F, seed):
    from paper_2505_14260_amd import mx
    g = gen(seed)
    x, y = (torch.randn(rows, d, generator=g).cuda() for _ in range(2))
    gain = (1 + 0.1 * torch.randn(d, generator=g)).bfloat16().cuda()
    wgu = (0.05 * torch.randn(2 * F, d, generator=g)).bfloat16().cuda()
    wd = (0.05 * torch.randn(d, F, generator=g)).bfloat16().cuda()
    qgu = mx.quantize(wgu, mx.MX(2 * F, d, layout="weight"))
    qd = mx.quantize(wd, mx.MX(d, F, layout="weight"))
    bufs = (torch.empty_like(x), mx.MX(rows, d), torch.empty(rows, 2 * F, device="cuda"),
            mx.MX(rows, F), torch.empty(rows, d, device="cuda"))
    return (x, y, gain, qgu, qd, bufs), (wgu, wd)


@pytest.mark.parametrize("rows, d, F", [(1, 128, 296), (10, 256, 688), (130, 512, 1000)])
def test_operators_together(rows, d, F):
    """An FFN: its output against the same chain in float64.  A rounding that falls
    the other way changes one value of a product's input by the two terms' error
    at most, top / 8 of its block; such blocks are under 1% (see near), so the
    result may differ by 1% of the blocks' worth, in norm 0.1 / 8 of its size."""
    args, (wgu, wd) = ffn_setup(rows, d, F, rows)
    x, y, gain = (t.double().cpu().numpy() for t in args[:3])
    out = ffn(*args).double().cpu().numpy()
    s = (x.astype(np.float32) + y.astype(np.float32)).astype(np.float64)
    a = O.quantised(O.rms_norm(s, gain, np.float64(np.float32(1e-5))), 2)
    gu = (a @ O.term(wgu.double().cpu().numpy()).T).astype(np.float32).astype(np.float64)
    ref = O.quantised(O.swiglu(gu[:, :F], gu[:, F:]), 2) @ O.term(wd.double().cpu().numpy()).T
    assert np.linalg.norm(out - ref) <= 0.1 / 8 * np.linalg.norm(ref)
    # and the 4-bit chain is near the unquantised one: two weights of 4 bits (12% each)
    # and two activations of two terms (1.5%)
    full = O.swiglu(*np.split(O.rms_norm(s, gain, 1e-5) @ wgu.double().cpu().numpy().T, 2, 1))
    full = full @ wd.double().cpu().numpy().T
    assert np.linalg.norm(out - full) <= 0.35 * np.linalg.norm(full)


def test_graph_replays_and_streams():
    """The chain captured once and replayed on new inputs, on a side stream, with
    eager work between the replays; repeats give the same bits."""
    args, _ = ffn_setup(20, 256, 688, 3)
    other, _ = ffn_setup(20, 256, 688, 4)
    x, y = args[0], args[1]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        ffn(*args)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = ffn(*args)
        for seed in range(4):
            x.copy_(torch.randn(x.shape, generator=gen(10 + seed)))
            y.copy_(torch.randn(x.shape, generator=gen(20 + seed)))
            graph.replay()
            got = out.clone()
            between = ffn(*other).clone()
            eager = ffn(*args).clone()
            stream.synchronize()
            assert torch.equal(got, eager)
            assert torch.equal(between, ffn(*other))
    torch.cuda.current_stream().wait_stream(stream)


def test_two_threads():
    """Calls of two threads, each on a stream of its own, at one time."""
    import threading
    jobs = [ffn_setup(rows, 256, 688, rows)[0] for rows in (20, 300)]
    want = [ffn(*args).clone() for args in jobs]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(50):
                    jobs[i][5][4].zero_()
                    if not torch.equal(ffn(*jobs[i]), want[i]):
                        wrong.append(i)
        except Exception as e:   # the thread's failure is the test's
            wrong.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not wrong and not any(t.is_alive() for t in threads)


def test_null_stream_entry_points():
    """The C calls on the null stream, from the raw binding."""
    from paper_2505_14260_amd import msd, mx
    x = torch.randn(5, 100, generator=gen(6)).cuda()
    q = mx.MX(5, 100)
    out = torch.empty(5, 100, device="cuda")
    torch.cuda.synchronize()
    msd.msd_mx_quantize(x.data_ptr(), msd.F32, 100, q.desc, None)
    msd.msd_mx_dequantize(q.desc, out.data_ptr(), msd.F32, 100, None)
    torch.cuda.synchronize()
    want = O.quantised(x.double().cpu().numpy(), 2).astype(np.float32)
    assert same(out.cpu().numpy(), want)
