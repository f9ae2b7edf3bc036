"""The first token drawn under a top_k whose border the oracle decides: it is one of those that
stay, and the one in whose interval the uniform number lies.

Logits of the GPU's target differ from the oracle's by delta, 2e-2 of the row's largest, at most:
weights at temperature T, and sums of them relative to the whole, by a factor e^(2 delta / T)."""
import math

import numpy as np
import pytest

from oracle import logits as OL
from test_gpu_logits_paths import prompt_logits, setup  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

pytest.importorskip("torch")


@pytest.mark.parametrize("top_k", [3, 7])
@pytest.mark.parametrize("T", [0.7, 1.0])
def test_the_token_is_the_one_at_the_uniform_numbers_place(setup, top_k, T):  # noqa: F811
    from paper_2505_14260_amd.msd import Sampling
    wl, eng, m, prompt, spec = setup
    z, delta = prompt_logits(m, prompt)
    ranked = -np.sort(-z)
    assert ranked[top_k - 1] - ranked[top_k] > 2 * delta      # the same tokens on the GPU
    ids, w, _ = OL.stay(z, temperature=T, top_k=top_k)
    kept = np.zeros(len(z))
    kept[ids] = w / w.sum()
    slack = math.expm1(2 * delta / T)
    drawn = []
    for u in np.linspace(0, 1 - 2.0 ** -24, 25):
        print(f"case: first of {top_k} tokens at {T}, u {u}", flush=True)
        t = eng.prefill(0, *prompt, sampling=Sampling(T, 1.0, 0.0, top_k), u=float(u))
        assert t in ids
        assert kept[:t].sum() - slack <= u <= kept[:t + 1].sum() + slack, (t, u)
        drawn.append(t)
    assert drawn == sorted(drawn) and len(set(drawn)) == top_k     # in the order of the ids, each met
