"""The operators on logits where the engine calls them: a sampled first token, acceptance
from a filtered distribution, and training from a teacher's record.

Logits of the GPU's target differ from the oracle's by 2e-2 of the row's largest at most
(the bound of every parity test): a probability at temperature T by a factor
e^(2 delta / T), delta that bound, and a running sum of them by as much.
"""
import math

import numpy as np
import pytest

import synth
from synth.configs import TINY
from oracle import logits as OL
from oracle import msd as O
from oracle import train as TR
from parity import sampling_agrees
from test_gpu_tiny import oracle_tree_from

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def setup():
    from paper_2505_14260_amd.msd import Engine, make_static_spec
    wl = TINY
    w = synth.make_target_weights(wl.dims, wl.seed)
    dr = synth.make_draft_weights(wl.dims, w, wl.seed, "random")
    eng = Engine(wl.dims, w, dr, max_batch=2, max_seq=256, max_tree=64,
                 max_prompt=max(wl.prompt_len, 64))
    parent, rank, _ = synth.static_tree_arrays(wl.tree.paths)
    yield wl, eng, O.Models(wl.dims, w, dr), synth.make_prompt(wl), make_static_spec(parent[1:], rank[1:])
    eng.close()


def prompt_logits(m, prompt):
    """The oracle's log-probabilities of a prompt's first token, and their error's bound."""
    from oracle import model as M
    h, _, pt = TR.sequence_inputs(m, *prompt)
    z = h[-1] @ np.asarray(M.widen(m.w["lm_head"]), dtype=np.float64).T
    return z, 2e-2 * np.abs(z).max()


@pytest.mark.parametrize("how", [
    dict(), dict(temperature=0.7, top_k=20), dict(top_p=0.8), dict(top_k=300, top_p=0.9, min_p=0.01)],
    ids=str)
def test_first_token_is_drawn(setup, how):
    from paper_2505_14260_amd.msd import Sampling
    wl, eng, m, prompt, spec = setup
    z, delta = prompt_logits(m, prompt)
    T = how.get("temperature", 1.0)
    s = Sampling(T, how.get("top_p", 1.0), how.get("min_p", 0.0), how.get("top_k", 0))
    p = np.exp((z - z.max()) / T)
    slack = math.expm1(2 * delta / T)
    ids, wts, _ = OL.stay(z, **how)
    worst = p[ids].min()           # a token that stays on the GPU is no less likely than about that
    trees = eng.new_trees(1)
    for u in (0.0, 0.03, 0.2, 0.41, 0.6, 0.83, 0.97, 1 - 2.0 ** -24):
        print(f"case: first token, {how}, u {u}", flush=True)
        t = eng.prefill(0, *prompt, sampling=s, u=u)
        assert p[t] >= worst * math.exp(-4 * delta / T)
        kept = np.zeros(len(z))
        kept[ids] = wts / wts.sum()
        lo, hi = kept[:t].sum(), kept[:t + 1].sum()
        if not how:                # nothing removed: the place of u itself
            assert lo - slack <= u <= hi + slack, (t, lo, hi, u, slack)
        eng.draft_tree([0], spec, trees)    # the drawn token is the tree's root
        assert eng.trees_to_host(trees, 1)[0].token[0] == t


def test_greedy_settings_are_the_greedy_decode(setup):
    """temperature 0, or one token that stays: the first token and whole answers are
    the greedy ones (speculative sampling of a point mass)."""
    from paper_2505_14260_amd.msd import Sampling
    wl, eng, m, prompt, spec = setup
    print("case: greedy settings", flush=True)
    want, _ = eng.generate(0, prompt, spec, 24)
    for s in (Sampling(0.0, 1.0, 0.0, 0), Sampling(1.0, 1.0, 0.0, 1), Sampling(1.0, 1e-9, 0.0, 0),
              Sampling(0.5, 1.0, 1.0, 0)):
        assert eng.prefill(0, *prompt, sampling=s, u=0.9) == want[0]
    for how in (dict(top_k=1), dict(top_p=1e-9), dict(min_p=1.0)):
        got, _ = eng.generate(0, prompt, spec, 24, temperature=1.0, seed=5, sample_first=True, **how)
        assert got == want, how


def test_filtered_acceptance_matches_oracle(setup):
    from oracle import sampling as S
    from paper_2505_14260_amd.msd import msd_seq_len
    wl, eng, m, prompt, spec = setup
    T = spec.n_nodes + 1
    trees = eng.new_trees(1)
    eng.prefill(0, *prompt)
    hows = [dict(top_k=5), dict(top_p=0.7), dict(min_p=0.2), dict(top_k=290, top_p=0.9, min_p=0.001)]
    for cyc in range(8):
        how, temp = hows[cyc % 4], (0.6, 1.1)[cyc // 4]
        print(f"case: filtered acceptance, {how} at {temp}", flush=True)
        eng.draft_tree([0], spec, trees)
        amax, logits = eng.verify([0], trees, T, want_logits=True)
        L = msd_seq_len(eng.ctx, 0)
        tree = oracle_tree_from(eng.trees_to_host(trees, 1)[0], T)
        lg = logits.cpu().numpy().reshape(T, -1)
        em, slots = eng.accept_sample([0], trees, T, logits, temp, 99, want_slots=True, **how)
        assert np.array_equal(logits.cpu().numpy().reshape(T, -1), lg)     # left as they were
        flt = np.full_like(lg, -np.inf)
        for r in range(T):
            ids, _, margin = OL.stay(lg[r], temperature=temp, **how)
            assert margin > 1e-9
            flt[r, ids] = lg[r, ids]
        n = len(em[0])
        path = [int(x) - L for x in slots.cpu().numpy()[:n]]
        r_path, r_emit, dec = S.sample_accept(tree, flt, temp, 99, 0, L)
        assert sampling_agrees(path, em[0], r_path, r_emit, dec), (cyc, path, r_path, em, r_emit)
        for node, token in zip(path, em[0]):        # each of them is one that stays at its node
            assert np.isfinite(flt[node, token])


def test_a_rejection_of_all_that_stays_emits_one_of_it(setup):
    """Two tokens stay and both are drafted.  In 32 bits 1 - p(first) can be more than
    p(second), so that the second may be rejected too, though all the mass left is its."""
    from oracle import sampling as S
    from paper_2505_14260_amd.msd import msd_seq_len
    wl, eng, m, prompt, spec = setup
    T = spec.n_nodes + 1
    print("case: both of the tokens that stay rejected", flush=True)
    trees = eng.new_trees(1)
    eng.prefill(0, *prompt)
    eng.draft_tree([0], spec, trees)
    _, logits = eng.verify([0], trees, T, want_logits=True)
    L = msd_seq_len(eng.ctx, 0)
    tree = eng.trees_to_host(trees, 1)[0]
    a, b = [int(tree.token[u]) for u in range(1, T) if tree.parent[u] == 0][:2]
    lg = torch.full((T, wl.dims.vocab), float("-inf"))
    lg[0, a] = 0.0
    lg[0, b] = math.log(0.55 * 2.0 ** -23)  # p(first) rounds to 1 - 2^-23
    seed = None
    for base in range(0, 1 << 28, 1 << 22):
        with np.errstate(over="ignore"):
            def uniform(j, seeds):
                z = seeds + np.uint64((S.draw_index(0, L, j) + 1) * S._GAMMA & S._M64)
                z = (z ^ z >> np.uint64(30)) * np.uint64(0xBF58476D1CE4E5B9)
                z = (z ^ z >> np.uint64(27)) * np.uint64(0x94D049BB133111EB)
                return (z ^ z >> np.uint64(31)) >> np.uint64(40)
            seeds = np.arange(base, base + (1 << 22), dtype=np.uint64)
            seeds = seeds[uniform(0, seeds) >= (1 << 24) - 2]
            seeds = seeds[uniform(1, seeds) >= 0.6 * (1 << 24)]
        if len(seeds):
            seed = int(seeds[0])
            break
    assert S.draw_uniform(seed, 0, L, 0) >= 1 - 2.0 ** -23 and S.draw_uniform(seed, 0, L, 1) >= 0.6
    em, _ = eng.accept_sample([0], trees, T, lg.cuda(), 1.0, seed)
    assert [int(x) for x in em[0]] == [b]


def test_settings_are_refused(setup):
    from paper_2505_14260_amd.msd import MSDError, Sampling
    wl, eng, m, prompt, spec = setup
    for bad in ((-1.0, 1.0, 0.0, 0), (float("nan"), 1.0, 0.0, 0), (1.0, 0.0, 0.0, 0), (1.0, 1.1, 0.0, 0),
                (1.0, 1.0, 2.0, 0), (1.0, 1.0, 0.0, -1)):
        with pytest.raises(MSDError):
            eng.prefill(0, *prompt, sampling=Sampling(*bad), u=0.5)


# --- training ------------------------------------------------------------------------------


def with_head_halved(m):
    """The oracle's models with an LM head of half the size: logits at temperature 2."""
    from oracle import model as M
    head = np.asarray(M.widen(m.w["lm_head"]), dtype=np.float32) / 2      # exact in bfloat16
    bits = (head.view(np.uint32) >> 16).astype(np.uint16)
    return O.Models(m.dims, dict(m.w, lm_head=bits), m.draft)


@pytest.mark.parametrize("k, T", [(1, 1.0), (16, 1.0), (200, 1.0), (64, 2.0)])
def test_training_from_a_record_matches_oracle(k, T):
    from paper_2505_14260_amd.msd import Engine
    wl = TINY
    print(f"case: training from a record of {k} at temperature {T}", flush=True)
    w = synth.make_target_weights(wl.dims, wl.seed)
    dr = synth.make_draft_weights(wl.dims, w, wl.seed, "random")
    m = O.Models(wl.dims, w, dr)
    eng = Engine(wl.dims, w, dr, max_seq=256, max_tree=64, max_prompt=max(wl.prompt_len, 64))
    try:
        prompts = [synth.make_prompt(wl, seq=0), synth.make_prompt(wl, seq=1)]
        cut = wl.n_visual + 7
        prompts[1] = tuple(a[:cut] for a in prompts[1][:2]) + (prompts[1][2],)
        seqs, loss, entropy = [], np.zeros(3), 0.0
        for p in prompts:
            ids, values = eng.train_record(0, *p, k=k)
            loss += eng.train_accumulate(0, *p, teacher=(ids, values, T))
            ids, values = ids.cpu().numpy(), values.double().cpu().numpy()
            h, e, pt = TR.sequence_inputs(m, *p)
            # the record is the target's: its largest logits, within their error
            z = np.log(pt[1:])
            got = values - values[:, :1]
            want = np.take_along_axis(z, ids, 1) - np.take_along_axis(z, ids[:, :1], 1)
            lm = np.abs(values).max()
            assert np.abs(got - want).max() <= 4e-2 * lm
            best = -np.sort(-z, 1)[:, :k]
            assert (np.take_along_axis(z, ids, 1) >= best - 4e-2 * lm).all()
            # the oracle's loss against the softmax of the record
            q = np.exp(got / T)
            q /= q.sum(1, keepdims=True)
            dense = np.zeros_like(pt)
            np.put_along_axis(dense[1:], ids, q, 1)
            entropy -= (q * np.log(q)).sum()
            seqs.append((h, e, p[1], dense))
        g = eng.train_read(0)
        rows = sum(len(p[0]) - 1 for p in prompts)
        mm = m if T == 1.0 else with_head_halved(m)
        _, reg, cls, gref = TR.batch_grads(mm, TR.draft_params(m.draft), seqs)
        kl = cls - entropy / rows
        assert abs(loss[1] / rows - reg) <= 1e-2 * reg
        assert abs(loss[2] / rows - kl) <= 1e-2 * cls, (loss[2] / rows, kl, cls)
        # the weight 0.1 is a float32: off by 2^-24 of itself at most (1.5e-9 here)
        assert abs(loss[0] - loss[1] - TR.CLS_WEIGHT * loss[2]) <= 2.0 ** -24 * TR.CLS_WEIGHT * abs(loss[2])
        for key in TR.PARAM_KEYS:
            err = np.abs(g[key] / rows - gref[key]).max() / np.abs(gref[key]).max()
            assert err <= 2e-2, (key, err)
    finally:
        eng.close()


def test_record_and_training_refusals(setup):
    from paper_2505_14260_amd import msd
    wl, eng, m, prompt, spec = setup
    tokens, vis, visual = prompt
    n = len(tokens)
    ids = torch.zeros(n - 1, 4, dtype=torch.int32, device="cuda")
    v = torch.zeros(n - 1, 4, device="cuda")
    for bad in ((ids[:-1], v[:-1], 1.0), (ids.long(), v, 1.0), (ids, v.half(), 1.0), (ids, v[:, :3], 1.0),
                (ids.cpu(), v, 1.0), (ids.t().contiguous().t(), v, 1.0)):
        with pytest.raises(ValueError):
            eng.train_accumulate(0, *prompt, teacher=bad)
    for T in (0.0, -1.0, float("nan"), 1e7):
        with pytest.raises(msd.MSDError):
            eng.train_accumulate(0, *prompt, teacher=(ids, v, T))
    for k in (0, 257):
        with pytest.raises(msd.MSDError):
            eng.train_record(0, *prompt, k=k)
    with pytest.raises(msd.MSDError):
        msd.msd_train_accumulate_top(eng.ctx, 0, tokens, vis, None, msd.Teacher(None, v.data_ptr(), 4, 1.0))
    for call in (lambda: msd.msd_train_record(None, 0, tokens, vis, None, 4, 4096, 4096, None),
                 lambda: msd.msd_prefill_sample(None, 0, tokens, vis, None,
                                                msd.Sampling(1.0, 1.0, 0.0, 0), 0.5)):
        with pytest.raises(msd.MSDError):
            call()


def test_all_of_them_together(setup):
    """Recorded once, trained from the record, then an answer sampled with the filters
    and the log-probabilities of its last verification."""
    from paper_2505_14260_amd import logits as L
    wl, eng, m, prompt, spec = setup
    print("case: record, train, sample, log-probabilities", flush=True)
    record = eng.train_record(1, *prompt, k=32)
    losses = []
    for _ in range(2):
        losses.append(eng.train_accumulate(1, *prompt, teacher=record + (1.0,)))
        eng.train_apply(1e-4)
    assert all(np.isfinite(x).all() for x in losses) and losses[0] != losses[1]
    how = dict(temperature=0.8, top_k=40, top_p=0.95, min_p=0.01)
    a, _ = eng.generate(0, prompt, spec, 20, seed=3, sample_first=True, **how)
    b, _ = eng.generate(0, prompt, spec, 20, seed=3, sample_first=True, **how)
    assert a == b and len(a) == 20 and all(0 <= t < wl.dims.vocab for t in a)
    T = spec.n_nodes + 1
    trees = eng.new_trees(1)
    eng.draft_tree([0], spec, trees)
    amax, logits = eng.verify([0], trees, T, want_logits=True)
    v = torch.empty(T, 5, device="cuda")
    i = torch.empty(T, 5, dtype=torch.int32, device="cuda")
    lse = torch.empty(T, device="cuda")
    L.top(logits, v, i, lse)
    assert torch.equal(i[:, 0], amax.view(-1))
    lp = torch.log_softmax(logits.double(), 1).gather(1, i.long())
    # 32-bit: the value, the lse and their difference round once each, the sum by 2^-18
    assert ((v - lse[:, None]).double() - lp).abs().max() <= 3 * 2.0 ** -24 * 30 + 2.0 ** -18
