"""What the operators on logits refuse, before any device work (no GPU).
Pointers are made up: a refused call reads none of them."""
import os

import pytest

from paper_2505_14260_amd import msd

if not os.path.exists(msd.LIB_PATH):
    pytest.skip("libmsd.so not built", allow_module_level=True)

X, Y, A, B, C, D, E = (0x100000000 * (i + 1) for i in range(7))
R, V, K = 4, 100, 8


def refused(call):
    with pytest.raises(msd.MSDError) as e:
        call()
    assert e.value.code == msd.MSD_ERR_INVALID_ARG and str(e.value).strip()
    assert msd.msd_last_error(None)


def how(temperature=1.0, top_p=1.0, min_p=0.0, top_k=0):
    return msd.Sampling(temperature, top_p, min_p, top_k)


def top(x=X, t=0, ld=V, rows=R, cols=V, k=K, values=A, ids=B, lse=C):
    msd.msd_logits_top(x, t, ld, rows, cols, k, values, ids, lse, None)


def sample(x=X, t=0, ld=V, rows=R, cols=V, s=None, u=A, tokens=B, lp=C):
    msd.msd_logits_sample(x, t, ld, rows, cols, s or how(), u, tokens, lp, None)


def filter_(x=X, t=0, ld=V, rows=R, cols=V, s=None, out=Y, ldo=V, kept=A):
    msd.msd_logits_filter(x, t, ld, rows, cols, s or how(), out, ldo, kept, None)


def distill(x=X, t=0, ld=V, rows=R, cols=V, ids=A, values=B, k=K, T=1.0, loss=C, lse=D, grad=E,
            dx=Y, ldd=V):
    msd.msd_logits_distill(x, t, ld, rows, cols, msd.Teacher(ids, values, k, T), loss, lse, grad, dx,
                           ldd, None)


CALLS = [top, sample, filter_, distill]


@pytest.mark.parametrize("call", CALLS, ids=lambda c: c.__name__)
@pytest.mark.parametrize("bad", [
    dict(x=None), dict(x=X + 2), dict(t=3), dict(t=-1), dict(ld=V - 1), dict(ld=1 << 60), dict(rows=-1),
    dict(rows=(1 << 21) + 1), dict(cols=0), dict(cols=-1), dict(cols=(1 << 18) + 1, ld=1 << 19),
    dict(x=X + 1, t=1)], ids=str)
def test_bad_logits(call, bad):
    refused(lambda: call(**bad))


@pytest.mark.parametrize("call, bad", [
    (top, dict(k=0)), (top, dict(k=-1)), (top, dict(k=257, cols=300, ld=300)), (top, dict(k=V + 1)),
    (top, dict(values=None)), (top, dict(ids=None)), (top, dict(values=A + 2)), (top, dict(lse=C + 1)),
    (sample, dict(u=None)), (sample, dict(tokens=None)), (sample, dict(lp=C + 2)),
    (filter_, dict(out=None)), (filter_, dict(ldo=V - 1)), (filter_, dict(out=Y + 2)),
    (filter_, dict(kept=A + 3)),
    (distill, dict(k=0)), (distill, dict(k=257)), (distill, dict(ids=None)), (distill, dict(values=None)),
    (distill, dict(T=0.0)), (distill, dict(T=9e-7)), (distill, dict(T=1.1e6)), (distill, dict(T=-1.0)), (distill, dict(T=float("inf"))),
    (distill, dict(T=float("nan"))), (distill, dict(grad=None)), (distill, dict(dx=None)),
    (distill, dict(loss=None, lse=None, grad=None, dx=None)), (distill, dict(ldd=V - 1)),
    (distill, dict(dx=Y + 1))], ids=lambda v: v.__name__ if callable(v) else str(v))
def test_bad_arrays_and_numbers(call, bad):
    refused(lambda: call(**bad))


@pytest.mark.parametrize("bad", [
    dict(temperature=-0.5), dict(temperature=float("inf")), dict(temperature=float("nan")),
    dict(top_p=0.0), dict(top_p=-0.1), dict(top_p=1.1), dict(top_p=float("nan")), dict(min_p=-0.1),
    dict(min_p=1.5), dict(min_p=float("nan")), dict(top_k=-1)], ids=str)
def test_bad_settings(bad):
    refused(lambda: sample(s=how(**bad)))
    refused(lambda: filter_(s=how(**bad)))


def test_null_settings():
    for c in (lambda: msd.msd_logits_sample(X, 0, V, R, V, None, A, B, C, None),
              lambda: msd.msd_logits_filter(X, 0, V, R, V, None, Y, V, A, None),
              lambda: msd.msd_logits_distill(X, 0, V, R, V, None, C, D, E, Y, V, None)):
        refused(c)


def test_calls_without_rows_are_checked_too_but_need_no_buffers():
    for call in (lambda **a: top(x=None, rows=0, values=None, ids=None, lse=None, **a),
                 lambda **a: sample(x=None, rows=0, u=None, tokens=None, lp=None, **a),
                 lambda **a: filter_(x=None, rows=0, out=None, kept=None, **a),
                 lambda **a: distill(x=None, rows=0, ids=None, values=None, loss=None, lse=None,
                                     grad=None, dx=None, **a)):
        refused(lambda: call(ld=V - 1))
        refused(lambda: call(t=9))


def test_overlaps():
    end = X + (R * V - 1) * 4   # the last logit
    refused(lambda: top(values=end))
    refused(lambda: top(ids=end))
    refused(lambda: top(lse=X))
    refused(lambda: top(ids=A + 4 * (R * K - 1)))
    refused(lambda: sample(tokens=end))
    refused(lambda: sample(tokens=A))
    refused(lambda: sample(lp=B + 4 * (R - 1)))
    refused(lambda: filter_(out=X + 4))                    # shifted, or otherwise strided
    refused(lambda: filter_(out=X, ldo=V + 1))
    refused(lambda: filter_(kept=end))
    refused(lambda: filter_(out=X, kept=end))              # in place as well
    refused(lambda: filter_(kept=Y + 8))
    refused(lambda: distill(dx=X + 4))
    refused(lambda: distill(dx=X, ldd=V + 2))
    refused(lambda: distill(dx=X, loss=end))
    refused(lambda: distill(dx=A))
    refused(lambda: distill(dx=B - 4))
    refused(lambda: distill(dx=E))
    refused(lambda: distill(loss=A))
    refused(lambda: distill(lse=C))
    refused(lambda: distill(loss=E))


def test_tensor_checks():
    torch = pytest.importorskip("torch")
    from paper_2505_14260_amd import logits as L
    x = torch.zeros(4, 100)
    f, i = torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    v, n = torch.zeros(4, 8), torch.zeros(4, 8, dtype=torch.int32)
    for call in (
            lambda: L.top(x[0], v, n), lambda: L.top(x, v[:3], n), lambda: L.top(x, v, n[:, :7]),
            lambda: L.top(x, v, n.long()), lambda: L.top(x.double(), v, n), lambda: L.top(x, v, None),
            lambda: L.top(x, None, n), lambda: L.top(x.t().contiguous().t(), v, n),
            lambda: L.top(x, v, n, f[:3]), lambda: L.sample(x, f.double(), i),
            lambda: L.sample(x, None, i), lambda: L.sample(x, f, None), lambda: L.sample(x, f[:3], i),
            lambda: L.sample(x, f, i, i), lambda: L.filter(x, x.bfloat16()),
            lambda: L.filter(x, torch.zeros(4, 99)), lambda: L.filter(x, x.clone(), f),
            lambda: L.distill(x, n, v[:, :7], 1.0, f), lambda: L.distill(x, n[:3], v[:3], 1.0, f),
            lambda: L.distill(x, None, v, 1.0, f), lambda: L.distill(x, n, v.double(), 1.0, f),
            lambda: L.distill(x, n, v, 1.0, f, None, f, x.half()),
            lambda: L.distill_backward(x, n, v, 1.0, None, x),
            lambda: L.distill_backward(x, n, v, 1.0, f, None),
            # right in all but that they are not on a GPU
            lambda: L.top(x, v, n, f), lambda: L.sample(x, f, i, f.clone()),
            lambda: L.filter(x, x.clone(), i), lambda: L.distill(x, n, v, 1.0, f),
            lambda: L.distill_backward(x, n, v, 1.0, f, x.clone())):
        with pytest.raises(ValueError):
            call()
