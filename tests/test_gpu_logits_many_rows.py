"""The operators on logits with more rows than the chip has compute units, for which other
kernels are launched than for a few: a few distinct rows repeated.  Each distinct row is
compared with the float64 oracle, every repeat with its first bit by bit.  The tolerances are
those counted in test_gpu_logits.py, which hold for 256 threads a row and more.

How many rows lie too near a border to be compared is bounded: a border of a row of V tokens
has one of the others within (V + 4) 2^-44 with a probability of about V times that, 0.4% at
2^18, so that of the nine rows of a case more than two are not to be met with."""
import numpy as np
import pytest

from oracle import logits as O
from test_gpu_logits import HALF_STEP, LAYOUTS, TYPES, U, f32, gen, host, i32, record, rows_of, strided, \
    sum_error

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROWS = 259
# of more than 32 KB in every type but the first, which is so in float32 alone
COLS = [8193, 16400, 32000, 50021, 152064, 262144]


def repeated(t):
    return t[torch.arange(ROWS) % t.shape[0]]


def first_of(t, n):
    """The first n rows, to which all the others are equal (NaN to NaN)."""
    head = t[:n]
    again = head[torch.arange(ROWS, device=t.device) % n]
    assert ((t == again) | ((t != t) & (again != again))).all()
    return head


def distinct(cols, type_, seed):
    """Rows as a head leaves them, and rows at which a choice can go wrong."""
    g = gen(seed)
    x = rows_of(9, cols, seed)
    x[3] = (x[3] * 2).round() / 2                               # very many equal ones
    x[4] = float("-inf")
    x[4, torch.randperm(cols, generator=g)[:300]] = torch.randn(300, generator=g) * 3
    x[5] = float("-inf")
    x[6] = torch.finfo(TYPES[type_]).min
    x[7, cols - 9:] = 40 + torch.arange(9) * 0.25               # the largest at the end
    x[8, ::3] = float("nan")
    return x.to(TYPES[type_])


@pytest.mark.parametrize("type_", list(TYPES))
def test_top_of_many_rows(type_):
    from paper_2505_14260_amd import logits as L
    for n, cols in enumerate(COLS):
        x = distinct(cols, type_, n)
        xs = strided(repeated(x.cuda()), *LAYOUTS[n % 3])
        for k in (1, 50, 64, 128, 256):
            print(f"case: top, {ROWS} x {cols} {type_}, k {k}", flush=True)
            v, i, lse = f32(ROWS, k), i32(ROWS, k), f32(ROWS)
            L.top(xs, v, i, lse)
            v, i, lse = (first_of(t, len(x)) for t in (v, i, lse))
            xh, v, i, lse = host(x), host(v), i.cpu().numpy(), host(lse)
            for r in range(len(x)):
                want_v, want_i, want = O.top(xh[r], k)
                assert np.array_equal(i[r], want_i) and np.array_equal(v[r], want_v), (r, k)
                if np.isinf(want):
                    assert lse[r] == want
                else:
                    row = np.where(np.isnan(xh[r]), -np.inf, xh[r])
                    assert abs(lse[r] - want) <= sum_error(row, 1.0)[0] + U * abs(want), (r, lse[r], want)


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("how", [
    dict(temperature=0.8, top_k=50, top_p=0.77731), dict(top_k=256), dict(), dict(top_p=0.77731),
    dict(temperature=1.5, top_p=0.98001, min_p=0.02), dict(min_p=0.05),
    dict(top_k=400, top_p=0.77731), dict(temperature=0.02, top_p=0.90001)], ids=str)
def test_choice_of_many_rows(how, type_):
    from paper_2505_14260_amd import logits as L
    for n, cols in enumerate(COLS):
        print(f"case: choice, {ROWS} x {cols} {type_}, {how}", flush=True)
        x = distinct(cols, type_, n)
        u = torch.rand(len(x), generator=gen(n))
        xs = strided(repeated(x.cuda()), *LAYOUTS[n % 3])
        out = strided(torch.zeros(ROWS, cols, dtype=x.dtype), *LAYOUTS[n % 3])
        kept, tokens, lp = i32(ROWS), i32(ROWS), f32(ROWS)
        L.filter(xs, out, kept, **how)
        L.sample(xs, repeated(u).cuda(), tokens, lp, **how)
        L.filter(xs, xs, **how)                                 # in place
        assert torch.equal(xs, out)
        out, kept, tokens, lp = (first_of(t, len(x)) for t in (out, kept, tokens, lp))
        xh, oh, lp = host(x), host(out), host(lp)
        kept, tokens = kept.cpu().numpy(), tokens.cpu().numpy()
        near, margin = 0, (cols + 4) * 2.0 ** -44
        for r in range(len(x)):
            ids, _, far = O.stay(xh[r], **how)
            token, logprob, far2 = O.sample(xh[r], float(u[r]), **how)
            assert (oh[r] > -np.inf).sum() == kept[r]
            if far < margin or far2 < margin:
                near += 1
                continue
            want = np.full(cols, -np.inf)
            want[ids] = xh[r][ids]
            assert kept[r] == len(ids), (r, kept[r], len(ids))
            assert np.array_equal(oh[r], want), r
            assert tokens[r] == token, (r, tokens[r], token)
            assert lp[r] == logprob or abs(lp[r] - logprob) <= U * abs(logprob) + margin, (r, lp[r], logprob)
        assert near <= 2, near


@pytest.mark.parametrize("type_", list(TYPES))
def test_distillation_of_many_rows(type_):
    """Loss alone, loss and gradient in one pass, and the same in the logits' place."""
    from paper_2505_14260_amd import logits as L
    for n, cols in enumerate(COLS):
        k, T = (16, 64, 256)[n % 3], (1.0, 2.0)[n % 2]
        print(f"case: distillation, {ROWS} x {cols} {type_}, k {k}, T {T}", flush=True)
        x = rows_of(8, cols, 40 + n)
        ids, v = record(x, k, n)
        x[1] = float("-inf")                                    # a mask, entries within it
        x[1, ids[1, ::2].long()] = 1.0
        v[1, 1::2] = float("-inf")
        ids[2] = -1
        ids[3, k // 2:] = ids[3, :k // 2].clone()               # every id twice
        ids[4, 3:] = cols
        x[5, ids[5, 0].long()] = float("-inf")                  # an infinite loss
        x[6] = float("-inf")
        x = x.to(TYPES[type_])
        g = 0.5 + torch.rand(len(x), generator=gen(n))
        xs = strided(repeated(x.cuda()), *LAYOUTS[n % 3])
        idd, vd, gd = repeated(ids).cuda(), repeated(v).cuda(), repeated(g).cuda()
        loss, lse, alone, placed = (f32(ROWS) for _ in range(4))
        dx = strided(torch.zeros(ROWS, cols, dtype=x.dtype), *LAYOUTS[n % 3])
        L.distill(xs, idd, vd, T, alone)
        L.distill(xs, idd, vd, T, loss, lse, gd, dx)
        L.distill(xs, idd, vd, T, placed, None, gd, xs)
        loss, lse, alone, placed, dx, xs = (first_of(t, len(x)) for t in (loss, lse, alone, placed, dx, xs))
        assert torch.equal(xs.nan_to_num(9.0), dx.nan_to_num(9.0))
        assert torch.equal(placed.nan_to_num(9.0), loss.nan_to_num(9.0))
        xh, dxh, loss, alone, lse, gh = host(x), host(dx), host(loss), host(alone), host(lse), host(g)
        for r in range(len(x)):
            want, wl, wdx, p, q = O.distill(xh[r], ids[r].numpy(), v[r].numpy(), T, gh[r])
            if np.isnan(want):
                assert np.isnan(loss[r]) and np.isnan(alone[r]) and np.isnan(dxh[r]).all(), r
                continue
            S, d = sum_error(xh[r], T)
            assert abs(lse[r] - wl) <= S + U * abs(wl), (r, lse[r], wl)
            for got in (loss[r], alone[r]):
                assert got == want or abs(got - want) <= S + U * abs(want) + 1e-12, (r, got, want, S)
            with np.errstate(invalid="ignore"):
                dev = np.where(p > 0, p * (S + (3 * d + 2) * U), 0) + 3 * U * (p + q)
            tol = gh[r] / T * dev + HALF_STEP[type_] * np.abs(wdx) + 2.0 ** -25 * (type_ == "f16") \
                + 2.0 ** -126
            bad = ~(np.abs(dxh[r] - wdx) <= tol)
            assert not bad.any(), (r, np.flatnonzero(bad)[:5], dxh[r][bad][:5], wdx[bad][:5], tol[bad][:5])


def test_training_from_a_record_of_many_rows():
    """A sequence of 300 rows at a vocabulary of 32,000, recorded and trained from: the
    gradient is written in the logits' place.  Bounds as for short sequences
    (test_gpu_logits_paths.py): losses to 1e-2, gradients to the 2e-2 of every parity test."""
    from dataclasses import replace

    import synth
    from synth.configs import TINY
    from oracle import msd as OM
    from oracle import train as TR
    from paper_2505_14260_amd.msd import Engine
    k = 64
    wl = replace(TINY, dims=replace(TINY.dims, vocab=32000), n_visual=230, n_text=70)
    n = wl.prompt_len
    print(f"case: training from a record of {k}, {n} rows", flush=True)
    w = synth.make_target_weights(wl.dims, wl.seed)
    dr = synth.make_draft_weights(wl.dims, w, wl.seed, "random")
    m = OM.Models(wl.dims, w, dr)
    eng = Engine(wl.dims, w, dr, max_seq=512, max_tree=64, max_prompt=n)
    try:
        p = synth.make_prompt(wl)
        record = eng.train_record(0, *p, k=k)
        loss = eng.train_accumulate(0, *p, teacher=record + (1.0,))
        g = eng.train_read(0)
        ids, values = record[0].cpu().numpy(), host(record[1])
        h, e, pt = TR.sequence_inputs(m, *p)
        z = np.log(pt[1:])
        lm = np.abs(values).max()
        got = values - values[:, :1]
        want = np.take_along_axis(z, ids, 1) - np.take_along_axis(z, ids[:, :1], 1)
        assert np.abs(got - want).max() <= 4e-2 * lm
        assert (np.take_along_axis(z, ids, 1) >= -np.sort(-z, 1)[:, :k] - 4e-2 * lm).all()
        q = np.exp(got)
        q /= q.sum(1, keepdims=True)
        dense = np.zeros_like(pt)
        np.put_along_axis(dense[1:], ids, q, 1)
        _, reg, cls, gref = TR.batch_grads(m, TR.draft_params(m.draft), [(h, e, p[1], dense)])
        kl = cls + (q * np.log(q)).sum() / (n - 1)
        assert abs(loss[1] / (n - 1) - reg) <= 1e-2 * reg
        assert abs(loss[2] / (n - 1) - kl) <= 1e-2 * cls, (loss[2] / (n - 1), kl, cls)
        for key in TR.PARAM_KEYS:
            err = np.abs(g[key] / (n - 1) - gref[key]).max() / np.abs(gref[key]).max()
            assert err <= 2e-2, (key, err)
    finally:
        eng.close()
