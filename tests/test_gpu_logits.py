"""The operators on rows of logits on the GPU against the float64 oracle (oracle/logits.py).

Order: values and ids of the top are exact.  What stays and what is drawn is exact
wherever no border is nearer than the operators' own rounding: weights are whole numbers
of 2^-45 of the largest, so a sum of V of them is off by V 2^-46 at most, and the
quotient of two sums, the larger at least 1, by twice that; the exponential is off by
2^-44 of itself at most, the quotient by twice that: (V + 4) 2^-44 covers them.
  log-probabilities: the same sum, and one rounding to float32.

Sums of 32-bit weights e^-d (log-sum-exp, loss, gradient), d = (max - x) / T.  A weight is
the product of the exponentials by which a thread's largest logit rose since, of the last
step to the row's, and its own: their arguments sum to d, each rounded with its difference
and with log2(e) / T (3 2^-24 of d together); each exponential is off by 2^-23 and its
product rounded (3 2^-24).  A thread of the 256 or 1024 of a row has units of 4 values or
more: at most V / 1024 + 1 rises, the last step and its own exponential, so 3 (V / 1024 + 3)
2^-24, and it adds its V / 256 + 8 values at most one by one; the rest is summed in 64
bits.  With D the mean of d under p a sum is off by
  S = (3 D + V / 64 + 18) 2^-24 relative
at most; lse and loss by S (their logarithm is taken in 64 bits) and one rounding of the
result; a p by S + (3 d + 2) 2^-24 of itself, and dx = g / T (p - q) by three more
roundings of either term and half a step of the output type.
"""
import numpy as np
import pytest

from oracle import logits as O

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
U = 2.0 ** -24


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rows_of(rows, cols, seed, bulk=2.0):
    """Logits: a bulk, and a few tokens far above it in some rows."""
    g = gen(seed)
    x = torch.randn(rows, cols, generator=g) * bulk
    at = torch.randint(0, cols, (rows, 12), generator=g)
    up = torch.rand(rows, 12, generator=g) * torch.rand(rows, 1, generator=g) * 12
    for r in range(rows):
        x[r, at[r]] = up[r]
    return x


def strided(x, pad=0, offset=0):
    """x on the GPU in rows `pad` values wider, `offset` values past the start."""
    rows, cols = x.shape
    buf = torch.full((rows * (cols + pad) + offset,), 77.0, dtype=x.dtype, device="cuda")
    v = buf[offset:].view(rows, cols + pad)[:, :cols]
    v.copy_(x)
    return v


def f32(*shape):
    return torch.full(shape, -5.0, device="cuda")


def i32(*shape):
    return torch.full(shape, -5, dtype=torch.int32, device="cuda")


def host(t):
    return t.double().cpu().numpy()


SIZES = [(1, 1), (1, 2), (3, 7), (2, 63), (5, 64), (4, 65), (2, 255), (3, 1000), (2, 1024), (2, 4095),
         (1, 4097), (2, 8193), (3, 32000), (1, 50021), (2, 65536), (1, 81920), (1, 81925), (1, 152064),
         (1, 163845), (1, 262144)]
LAYOUTS = [(0, 0), (8, 8), (3, 1)]


def sum_error(x, temperature):
    """S of the header, and d / T of every logit."""
    with np.errstate(invalid="ignore"):
        d = (x.max() - x) / temperature
        p = np.exp(-d)
        D = np.where(p > 0, p * d, 0).sum() / p.sum()
    return (3 * D + 18 + len(x) / 64) * U, d


# --- top -----------------------------------------------------------------------------------


def check_top(x, k):
    from paper_2505_14260_amd import logits as L
    R = x.shape[0]
    v, i, lse = f32(R, k), i32(R, k), f32(R)
    L.top(x, v, i, lse)
    xh, v, i, lse = host(x), host(v), i.cpu().numpy(), host(lse)
    for r in range(R):
        want_v, want_i, want = O.top(xh[r], k)
        assert np.array_equal(i[r], want_i) and np.array_equal(v[r], want_v), (r, k)
        if np.isinf(want):
            assert lse[r] == want
        else:
            row = np.where(np.isnan(xh[r]), -np.inf, xh[r])
            assert abs(lse[r] - want) <= sum_error(row, 1.0)[0] + U * abs(want), (r, lse[r], want)


@pytest.mark.parametrize("type_", list(TYPES))
def test_top(type_):
    for n, (rows, cols) in enumerate(SIZES):
        x = rows_of(rows, cols, n).to(TYPES[type_])
        for j, k in enumerate(sorted({1, min(10, cols), min(64, cols), min(256, cols)})):
            pad, offset = LAYOUTS[(n + j) % 3]
            print(f"case: {rows} x {cols}, k {k}, pad {pad}", flush=True)
            check_top(strided(x, pad, offset), k)


def test_top_ties_and_special_values():
    for cols in (5, 300, 5000, 40000):
        x = torch.randint(-3, 4, (14, cols), generator=gen(cols)).float()
        x[1] = 0                                         # all equal
        x[2] = float("-inf")                             # nothing
        x[3, 1:] = float("-inf")                         # one token
        x[4] = torch.where(torch.arange(cols) % 2 == 0, -0.0, 0.0)
        x[5, ::3] = float("nan")
        x[6] = float("nan")
        x[7, cols // 2] = float("inf")
        x[8] = torch.finfo(torch.float32).max
        x[9] = -torch.finfo(torch.float32).max
        x[10] = torch.arange(cols).flip(0) * 1e-45       # denormals, descending
        x[11] = torch.arange(cols) * 0.25                # the largest all at the end
        x[12, :] = float("-inf")
        x[12, cols // 2:] = 1.5
        x[13] = torch.where(torch.arange(cols) % 64 == 0, 5.0, -1.0)   # in one thread of each wave
        for k in sorted({1, 2, min(100, cols), min(256, cols)}):
            print(f"case: {cols} columns, k {k}", flush=True)
            check_top(x.cuda(), k)


# --- what stays, and what is drawn -----------------------------------------------------------


SETTINGS = [
    dict(), dict(temperature=0.0), dict(temperature=0.3), dict(temperature=2.5),
    dict(top_k=1), dict(top_k=50), dict(top_k=256), dict(top_k=257), dict(top_k=3000),
    dict(top_p=0.9), dict(top_p=0.999), dict(top_p=1e-6), dict(top_p=0.5, temperature=3.0),
    dict(min_p=0.05), dict(min_p=1.0), dict(min_p=1e-4, temperature=1.7),
    dict(temperature=0.8, top_k=50, top_p=0.9), dict(temperature=1.3, top_k=2000, top_p=0.95),
    dict(temperature=1.5, top_p=0.98, min_p=0.02), dict(top_k=40, min_p=0.1),
    dict(temperature=1e-3, top_p=0.9), dict(temperature=1e4, top_p=0.7),
    dict(temperature=0.7, top_k=20, top_p=0.8, min_p=0.05)]


def check_choice(x, u, how, layout=(0, 0)):
    """Returns how many rows were too near a border to be compared."""
    from paper_2505_14260_amd import logits as L
    R, V = x.shape
    x = strided(x, *layout)
    out = strided(torch.zeros(R, V, dtype=x.dtype), *layout)
    kept, tokens, lp = i32(R), i32(R), f32(R)
    assert L.filter(x, out, kept, **how) is out
    assert L.sample(x, u.cuda(), tokens, lp, **how) is tokens
    xh, oh = host(x), host(out)
    kept, tokens, lp = kept.cpu().numpy(), tokens.cpu().numpy(), host(lp)
    near = 0
    margin = (V + 4) * 2.0 ** -44
    for r in range(R):
        ids, _, far = O.stay(xh[r], **how)
        token, logprob, far2 = O.sample(xh[r], float(u[r]), **how)
        assert (oh[r] > -np.inf).sum() == kept[r]
        if far < margin or far2 < margin:
            near += 1
            continue
        want = np.full(V, -np.inf)
        want[ids] = xh[r][ids]
        assert kept[r] == len(ids), (r, how, kept[r], len(ids))
        assert np.array_equal(oh[r], want), (r, how)
        assert tokens[r] == token, (r, how, tokens[r], token)
        if np.isinf(logprob):
            assert lp[r] == logprob
        else:
            assert abs(lp[r] - logprob) <= U * abs(logprob) + (V + 4) * 2.0 ** -44
    return near


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("how", SETTINGS, ids=str)
def test_stay_and_sample(how, type_):
    near = total = 0
    for n, (rows, cols) in enumerate(SIZES):
        print(f"case: {rows} x {cols}", flush=True)
        x = rows_of(rows, cols, 100 + n).to(TYPES[type_])
        u = torch.rand(rows, generator=gen(n))
        near += check_choice(x, u, how, layout=LAYOUTS[n % 3])
        total += rows
    assert near <= total * 0.05, near


@pytest.mark.parametrize("how", [
    dict(), dict(temperature=0.0), dict(top_k=3), dict(top_k=1000), dict(top_p=0.3), dict(min_p=0.5),
    dict(top_k=100, top_p=0.7), dict(temperature=2.0, top_p=0.4, min_p=0.2)], ids=str)
def test_stay_special_rows(how):
    for cols in (1, 6, 700, 5000, 40000, 170000):
        print(f"case: {cols} columns", flush=True)
        x = torch.randint(-3, 4, (11, cols), generator=gen(cols)).float()
        x[0] = float("-inf")
        x[1] = float("nan")
        x[2] = 0
        x[3] = float("-inf")
        x[3, cols - 1] = -1e30
        x[4, ::2] = float("nan")
        x[4, cols // 2] = 9
        x[5, 0] = float("inf")
        x[5, cols - 1] = float("inf")
        x[6] = torch.finfo(torch.float32).max * torch.linspace(-1, 1, cols)
        x[7] = torch.where(torch.arange(cols) % 2 == 0, -0.0, 0.0)
        x[8] = torch.finfo(torch.float32).min
        u = torch.rand(11, generator=gen(3))
        check_choice(x, u, how)


@pytest.mark.parametrize("dead", ["-inf", "lowest"])
@pytest.mark.parametrize("how", [
    dict(), dict(top_k=30), dict(top_k=400), dict(top_p=0.8), dict(min_p=0.1),
    dict(top_p=0.9, min_p=0.01), dict(temperature=0.05, top_p=0.9), dict(temperature=40.0, top_p=0.5),
    dict(top_k=200, top_p=0.7)], ids=str)
def test_stay_masked_rows(how, dead):
    """A mask leaves a few tokens, anywhere: also where a row's first are masked."""
    for cols in (300, 5000, 40000, 152064):
        print(f"case: {cols} columns", flush=True)
        g = gen(cols)
        for type_ in ("f32", "bf16"):
            low = float("-inf") if dead == "-inf" else torch.finfo(TYPES[type_]).min
            x = torch.full((7, cols), low)
            for r, live in enumerate((1, 2, 20, 60, 250, 280, 300)):
                at = torch.randperm(cols, generator=g)[:live]
                x[r, at] = torch.randn(live, generator=g) * 3 + r
            x[5, : cols // 2] = low
            x[6, cols // 3:] = low
            check_choice(x.to(TYPES[type_]), torch.rand(7, generator=g), how)


def test_stay_with_a_late_maximum_and_odd_scales():
    """The largest far above what a row begins with, in units of the temperature; logits far
    from 0; temperatures at which all weigh alike."""
    for cols in (3000, 70000):
        g = gen(cols)
        x = torch.randn(8, cols, generator=g)
        x[0, cols - 1] = 30
        x[1, cols // 2:] += 25
        x[2] += 3000
        x[3] = x[3] * 1e-3 - 5e4
        x[4] *= 1e30
        x[5, cols - 5:] = torch.tensor([50.0, 49.9, 49.8, 49.7, 49.6])
        x[6] = torch.linspace(-80, 80, cols)
        x[7] = torch.linspace(80, -80, cols)
        u = torch.rand(8, generator=g)
        for how in (dict(temperature=0.02, top_p=0.9), dict(temperature=0.3, top_p=0.95, min_p=0.01),
                    dict(temperature=1.0, top_p=0.99), dict(temperature=1e-5, top_p=0.6),
                    dict(temperature=1e9, top_p=0.3), dict(temperature=1e45, top_p=0.75),
                    dict(temperature=2.0, min_p=0.3), dict(temperature=0.01, top_k=300, top_p=0.9)):
            print(f"case: {cols} columns, {how}", flush=True)
            check_choice(x, u, how)


def test_stay_with_a_top_k_of_more_than_a_mask_leaves():
    for cols, live in ((3000, 700), (40000, 2500)):
        g = gen(cols)
        x = torch.full((6, cols), float("-inf"))
        for r in range(6):
            at = torch.randperm(cols, generator=g)[:live + r]
            x[r, at] = torch.randn(live + r, generator=g) * (0.02 if r & 1 else 2) + r
        u = torch.rand(6, generator=g)
        for how in (dict(top_k=live + 90, top_p=0.9, min_p=0.5), dict(top_k=live + 90, top_p=0.5, min_p=0.1),
                    dict(top_k=live + 90, top_p=0.3, min_p=0.97), dict(top_k=live + 1, top_p=0.95)):
            print(f"case: {cols} columns, {how}", flush=True)
            check_choice(x, u, how)


def test_top_of_masked_rows():
    for cols in (300, 5000, 60000):
        x = torch.full((5, cols), float("-inf"))
        for r, live in enumerate((1, 9, 100, 255, 299)):
            at = torch.randperm(cols, generator=gen(r))[:live]
            x[r, at] = torch.randn(live, generator=gen(r + 9))
        for k in (1, 64, 100, 256):
            print(f"case: {cols} columns, k {k}", flush=True)
            check_top(x.cuda(), k)
            check_top(torch.where(x == float("-inf"), torch.finfo(torch.float32).min, x).cuda(), k)


def test_stay_with_exact_borders():
    """Weights that are powers of two sum exactly: a border may lie on a sum."""
    log2 = float(np.log(2.0))
    from paper_2505_14260_amd import logits as L
    for cols in (64, 4096, 65536):
        x = torch.full((1, cols), 1.25).cuda()          # equal: the lowest ids stay
        out, kept, tok = torch.empty_like(x), i32(1), i32(1)
        for p, want in ((0.5, cols // 2), (1 / cols, 1), (1.5 / cols, 2), (1 - 1 / cols, cols - 1)):
            L.filter(x, out, kept, top_p=p)
            assert kept.item() == want and (out[0, :want] == 1.25).all()
            assert (out[0, want:] == float("-inf")).all()
        for i in (0, 1, cols // 3, cols - 1):           # u on the border before id i
            L.sample(x, torch.tensor([i / cols]).cuda(), tok)
            assert tok.item() == i
        L.filter(x, out, kept, top_k=7)
        assert kept.item() == 7 and (out[0, :7] == 1.25).all()
    # weights 1, 1/2, 1/4, 1/4 with T = 1 / log 2: exp((x - max) / T) = 2^(x - max)
    x = torch.tensor([[-1.0, 0.0, -2.0, -2.0]]).cuda()
    out, kept = torch.empty_like(x), i32(1)
    for p, want in ((0.5, 1), (0.500001, 2), (0.75, 2), (0.76, 3), (0.875, 3), (0.9, 4)):
        L.filter(x, out, kept, temperature=1 / log2, top_p=p)
        assert kept.item() == want, (p, kept.item())
    for mp, want in ((0.5, 2), (0.4999, 2), (0.51, 1), (0.25, 4), (0.26, 2)):
        L.filter(x, out, kept, temperature=1 / log2 * (1 + 1e-12), min_p=mp)
        assert kept.item() == want, (mp, kept.item())


def test_sample_follows_the_probabilities():
    """u on a grid of N points draws a token N p times, give or take one."""
    from paper_2505_14260_amd import logits as L
    N, V = 4096, 500
    row = rows_of(1, V, 9)
    x = row.expand(N, V).contiguous().cuda()
    tok = i32(N)
    how = dict(temperature=0.9, top_k=60, top_p=0.97)
    L.sample(x, (torch.arange(N) / N).cuda(), tok, **how)
    ids, w, _ = O.stay(row[0].double().numpy(), **how)
    got = np.bincount(tok.cpu().numpy(), minlength=V)
    want = np.zeros(V)
    want[ids] = w / w.sum() * N
    assert (np.abs(got - want) <= 1 + 1e-6).all()


def test_sample_uniforms_at_and_past_the_ends():
    from paper_2505_14260_amd import logits as L
    x = rows_of(1, 3000, 4)
    last_first = (O.sample(x[0].double().numpy(), u)[0] for u in (0.0, 1 - 2.0 ** -24))
    first, last = last_first
    us = [0.0, -1.0, float("nan"), -0.0, 1 - 2.0 ** -24, 1.0, 2.0, float("inf"), -float("inf")]
    tok = i32(len(us))
    L.sample(x.expand(len(us), 3000).contiguous().cuda(), torch.tensor(us).cuda(), tok)
    tok = tok.cpu().tolist()
    assert tok[:4] == [first] * 4 and tok[8] == first and tok[4] == last
    live = O.weights(x[0].double().numpy(), 1.0)
    assert all(t == np.flatnonzero(live >= 2.0 ** -46)[-1] for t in tok[5:8])


# --- distillation ----------------------------------------------------------------------------


def record(x, k, seed):
    """A teacher's record of rows near x."""
    t = x.float() + torch.randn(x.shape, generator=gen(seed)) * 0.7
    v, i = torch.topk(t, k, dim=1)
    return i.to(torch.int32), v


def check_distill(x, ids, values, T, type_, layout=(0, 0), seed=0):
    from paper_2505_14260_amd import logits as L
    R, V = x.shape
    xs = strided(x, *layout)
    g = 0.5 + torch.rand(R, generator=gen(seed))
    loss, lse = f32(R), f32(R)
    dx, dx2 = (strided(torch.zeros(R, V, dtype=x.dtype), *layout) for _ in range(2))
    idd, vd, gd = ids.cuda(), values.cuda(), g.cuda()
    L.distill(xs, idd, vd, T, loss, lse, gd, dx)
    loss2 = f32(R)
    L.distill(xs, idd, vd, T, loss2)
    L.distill_backward(xs, idd, vd, T, gd, dx2)
    assert torch.equal(loss, loss2) or torch.isnan(loss).any()
    assert torch.equal(dx, dx2) or torch.isnan(dx).any()
    xh, dxh, loss, lse, gh = host(x), host(dx), host(loss), host(lse), host(g)
    for r in range(R):
        want, wl, wdx, p, q = O.distill(xh[r], ids[r].numpy(), values[r].numpy(), T, gh[r])
        S, d = sum_error(xh[r], T)
        if np.isnan(want):
            assert np.isnan(loss[r]) and np.isnan(dxh[r]).all(), r
            continue
        assert abs(lse[r] - wl) <= S + U * abs(wl), (r, lse[r], wl)
        if np.isinf(want):
            assert loss[r] == want
        else:
            # q log q and q log p in 64 bits from 1 / T rounded there
            assert abs(loss[r] - want) <= S + U * abs(want) + 1e-12, (r, loss[r], want, S)
        with np.errstate(invalid="ignore"):
            dev = np.where(p > 0, p * (S + (3 * d + 2) * U), 0) + 3 * U * (p + q)
        tol = gh[r] / T * dev + HALF_STEP[type_] * np.abs(wdx) + 2.0 ** -25 * (type_ == "f16") + 2.0 ** -126
        bad = ~(np.abs(dxh[r] - wdx) <= tol)
        assert not bad.any(), (r, np.flatnonzero(bad)[:5], dxh[r][bad][:5], wdx[bad][:5], tol[bad][:5])


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("T", [1.0, 2.0, 0.5])
def test_distill(type_, T):
    for n, (rows, cols) in enumerate(SIZES):
        x = rows_of(rows, cols, 200 + n).to(TYPES[type_])
        k = (1, 5, 64, 100, 256)[n % 5]
        ids, v = record(x, min(k, cols), n)
        print(f"case: {rows} x {cols}, k {ids.shape[1]}", flush=True)
        check_distill(x, ids, v, T, type_, LAYOUTS[n % 3], n)


def test_distill_special_rows():
    for cols in (9, 3000, 40000):
        x = rows_of(14, cols, cols)
        ids, v = record(x, 8, 1)
        ids[0] = -1                                       # no entries
        ids[1, 3:] = -1                                   # three
        ids[2, 2] = cols                                  # outside
        ids[2, 3] = 2 ** 31 - 1
        ids[3] = ids[3, 0].item()                         # one id eight times
        ids[4, 4:] = ids[4, :4].clone()                   # four ids twice
        v[5] = float("-inf")
        v[6, 1:] = float("-inf")
        v[7, 2] = float("nan")
        v[8, 2] = float("inf")
        x[9, ids[9, 0].long()] = float("-inf")            # infinite loss
        x[10, torch.arange(cols) % 2 == 1] = float("-inf")  # masked tokens, some with entries
        x[11, 1] = float("nan")
        x[12, 1] = float("inf")
        x[13] = float("-inf")
        v[0, 0] = float("nan")                            # of no entry: not looked at
        for T in (1.0, 3.0):
            print(f"case: {cols} columns, T {T}", flush=True)
            check_distill(x, ids, v, T, "f32")


def test_distill_gradient_against_differences():
    from paper_2505_14260_amd import logits as L
    x = rows_of(1, 40, 5, bulk=1.0)
    ids, v = record(x, 6, 2)
    dx = f32(1, 40)
    L.distill_backward(x.cuda(), ids.cuda(), v.cuda(), 1.5, torch.tensor([0.8]).cuda(), dx)
    h = 1e-5
    for c in range(40):
        lo, hi = x[0].double().numpy().copy(), x[0].double().numpy().copy()
        lo[c] -= h
        hi[c] += h
        d = (O.distill(hi, ids[0].numpy(), v[0].numpy(), 1.5)[0]
             - O.distill(lo, ids[0].numpy(), v[0].numpy(), 1.5)[0]) / (2 * h) * np.float32(0.8)
        # h^2 of the third derivative (at most 1 / T^3), 2^-52 / h of the difference, the operator's own
        assert abs(dx[0, c].item() - d) <= h * h + 2.0 ** -50 / h * 10 + 12 * U


# --- how they are called ---------------------------------------------------------------------


def run_all(x, u, ids, v, g, o):
    from paper_2505_14260_amd import logits as L
    how = dict(temperature=0.9, top_k=300, top_p=0.9, min_p=0.001)
    L.top(x, o["v"], o["i"], o["lse"])
    L.sample(x, u, o["tok"], o["lp"], **how)
    L.filter(x, o["out"], o["kept"], **how)
    L.distill(x, ids, v, 1.0, o["loss"], o["l2"], g, o["dx"])


def outputs(R, V, k=16, dtype=torch.float32):
    z = dict(dtype=dtype, device="cuda")
    return dict(v=f32(R, k), i=i32(R, k), lse=f32(R), tok=i32(R), lp=f32(R), out=torch.empty(R, V, **z),
                kept=i32(R), loss=f32(R), l2=f32(R), dx=torch.empty(R, V, **z))


def inputs(R, V, seed, dtype=torch.float32):
    x = rows_of(R, V, seed).to(dtype)
    ids, v = record(x, 16, seed)
    g = gen(seed + 1)
    return (x.cuda(), torch.rand(R, generator=g).cuda(), ids.cuda(), v.cuda(),
            torch.rand(R, generator=g).cuda())


def test_replayed_graphs_other_inputs_and_repeats():
    """Captured calls, replayed on new inputs between eager work, twice over."""
    R, V = 9, 33001
    ins = inputs(R, V, 0)
    o = outputs(R, V)
    run_all(*ins, o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run_all(*ins, o)
    for seed in (1, 2, 1):
        new = inputs(R, V, seed)
        want = outputs(R, V)
        run_all(*new, want)
        again = outputs(R, V)
        run_all(*new, again)
        for t, s in zip(ins, new):
            t.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        for n in o:
            assert torch.equal(o[n], want[n]) and torch.equal(again[n], want[n]), (seed, n)


def test_two_streams_at_once():
    R, V = 40, 32000
    ins = [inputs(R, V, s) for s in (0, 1)]
    want = [outputs(R, V) for _ in ins]
    for a, o in zip(ins, want):
        run_all(*a, o)
    got = [outputs(R, V) for _ in ins]
    streams = [torch.cuda.Stream() for _ in ins]
    torch.cuda.synchronize()
    for _ in range(3):
        for st, a, o in zip(streams, ins, got):
            with torch.cuda.stream(st):
                run_all(*a, o)
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        for n in w:
            assert torch.equal(w[n], g[n]), n


@pytest.mark.parametrize("type_", list(TYPES))
def test_in_place_and_what_lies_beside(type_):
    from paper_2505_14260_amd import logits as L
    for rows, cols in ((5, 999), (3, 40000), (2, 170001)):
        x, u, ids, v, g = inputs(rows, cols, 3, TYPES[type_])
        how = dict(top_p=0.8, temperature=1.2)
        want, wdx = torch.empty_like(x), torch.empty_like(x)
        L.filter(x, want, **how)
        L.distill_backward(x, ids, v, 1.0, g, wdx)
        for pad, offset in LAYOUTS + [(5, 3)]:
            buf = torch.full((offset + (rows + 1) * (cols + pad),), 7.0, dtype=x.dtype, device="cuda")
            y = buf[offset:].view(rows + 1, cols + pad)
            for call, w in ((lambda t: L.filter(t, t, **how), want),
                            (lambda t: L.distill_backward(t, ids, v, 1.0, g, t), wdx)):
                y[:rows, :cols] = x
                call(y[:rows, :cols])
                assert torch.equal(y[:rows, :cols], w)
                assert (y[:rows, cols:] == 7).all() and (y[rows] == 7).all() and (buf[:offset] == 7).all()


def test_no_rows_and_rows_of_one():
    from paper_2505_14260_amd import logits as L
    x = torch.empty(0, 50, device="cuda")
    run_all(x, f32(0), i32(0, 16), f32(0, 16), f32(0), outputs(0, 50))
    # a column of a matrix: one logit a row
    y = torch.randn(6, 4, generator=gen(0)).cuda()[:, 2:3]
    tok, v, i = i32(6), f32(6, 1), i32(6, 1)
    L.sample(y, torch.rand(6).cuda(), tok, top_p=0.5)
    L.top(y, v, i)
    assert (tok == 0).all() and (i == 0).all() and torch.equal(v, y)


def test_many_short_rows():
    R, V = 70001, 5
    x = rows_of(64, V, 6).cuda()
    from paper_2505_14260_amd import logits as L
    big = x.repeat(-(-R // 64), 1)[:R].contiguous()
    vals, idx, lse = f32(R, 5), i32(R, 5), f32(R)
    L.top(big, vals, idx, lse)
    want = [O.top(r, 5) for r in host(x)]
    wi = torch.tensor(np.array([w[1] for w in want]), dtype=torch.int32).repeat(-(-R // 64), 1)[:R]
    assert torch.equal(idx.cpu(), wi)
    out, kept = torch.empty_like(big), i32(R)
    L.filter(big, out, kept, top_k=2)
    assert (kept == 2).all() and torch.equal(out > float("-inf"), (
        torch.zeros_like(out, dtype=torch.bool).scatter_(1, idx[:, :2].long(), True)))


def test_offsets_past_32_bits():
    """Rows that begin beyond 2^32 bytes and 2^31 values."""
    from paper_2505_14260_amd import logits as L
    V, R = 120000, 18200   # 2.18e9 values
    x = torch.zeros(R, V, dtype=torch.bfloat16, device="cuda")
    tail = rows_of(3, V, 8).bfloat16().cuda()
    x[R - 3:] = tail
    v, i, w, j = f32(R, 9), i32(R, 9), f32(3, 9), i32(3, 9)
    L.top(x, v, i)
    L.top(tail, w, j)
    assert torch.equal(v[R - 3:], w) and torch.equal(i[R - 3:], j)
    assert (i[:R - 3] == torch.arange(9, device="cuda")).all()
    kept, want = i32(R), torch.empty_like(tail)
    L.filter(tail, want, top_p=0.9)
    L.filter(x, x, kept, top_p=0.9)
    assert torch.equal(x[R - 3:], want) and (kept[:R - 3] == 108000).all()
