"""The sampling oracle where everything that a filter keeps was drafted and rejected: in
floating point 1 - (mass rejected) may exceed the mass of the last token that is left, so
that its acceptance falls short of 1.  Then the last rejected token with mass is emitted,
as include/msd.h defines it."""
import numpy as np
import pytest

from oracle import sampling as S
from test_oracle_sampling import make_tree

LARGEST = 1 - 2.0 ** -24     # the largest uniform number


def all_rejected():
    """Logits that keep tokens 6, 2 and 4 (in the order of the children), and whose
    children are rejected one after the other by the largest uniform number."""
    for i in range(1, 64):
        p = np.zeros(8)
        p[2] = (2.0 ** -24 + 2.0 ** -40) * (1 - 2.0 ** -23)
        p[4] = 2.0 ** -47 * i / 64
        p[6] = 1 - 2.0 ** -24 - 2.0 ** -40
        with np.errstate(divide="ignore"):
            row = np.log(p)
        q = S.target_probs(row, 1.0)
        removed, ok = 0.0, True
        for x in (6, 2, 4):
            ok = ok and LARGEST >= q[x] / (1.0 - removed)
            removed += q[x]
        if ok:
            return row
    raise AssertionError("no such row")


@pytest.mark.parametrize("masked", [(), (0,)])
def test_the_last_rejected_token_with_mass_is_emitted(monkeypatch, masked):
    monkeypatch.setattr(S, "draw_uniform", lambda seed, seq, L, j: LARGEST)
    row = all_rejected()
    token = [1, 6, 2, 4] + list(masked)      # a masked child after them has no mass
    tree = make_tree([-1] + [0] * (len(token) - 1), token)
    path, emitted, decisions = S.sample_accept(tree, np.tile(row, (len(token), 1)), 1.0, 0, 0, 0)
    assert [d["kind"] for d in decisions] == ["child"] * (len(token) - 1) + ["bonus"]
    assert path == [0] and emitted == [4]


def test_a_token_that_stays_comes_before_a_rejected_one(monkeypatch):
    """Of zero mass in 64 bits, but not masked."""
    monkeypatch.setattr(S, "draw_uniform", lambda seed, seq, L, j: LARGEST)
    row = all_rejected()
    row[7], row[3] = -800.0, -900.0
    tree = make_tree([-1, 0, 0, 0], [1, 6, 2, 4])
    assert S.sample_accept(tree, np.tile(row, (4, 1)), 1.0, 0, 0, 0)[1] == [7]
