"""The draft in 4 bits (msd_set_draft_mx) against the float64 oracle with the same
roundings: every product of the draft takes its weight as 4-bit blocks and its input
in two 4-bit terms (oracle/mx.py), everything else is the oracle's draft.

Tolerances.  A rounding to 4 bits is a step function: where the GPU's input and the
oracle's lie on two sides of a border, the rounded values differ by a step.  Both lie
within the rounding's error E of nearly the same input, so the results of a product
differ by at most 2 E of their norm (the weights are random: they keep the ratio of
norms), E being the largest relative error, in the 2-norm of a row, of the oracle's own
roundings of two terms (1.5% for normal values; without the second term 11.5%).
  - draft keys and values behind f_down and the q/k/v product: 4 E of a row's norm;
  - rows whose rounded inputs are exact (visual embeddings; an imported bfloat16
    feature): the float32 norm puts 1 value in 2^17 on the other side, and the cache is
    bfloat16: 2^-7 of the row's largest magnitude, as for the bfloat16 draft;
  - logits, behind six products whose roundings are independent: 2 E sqrt(6) of the
    row's largest magnitude decides between tokens (tests/parity.py's rule).
"""
import contextlib
import dataclasses

import numpy as np
import pytest

import synth
from synth.configs import TINY, WIDE
from oracle import model as M
from oracle import msd as O
from oracle import mx
from parity import (argmax_ok, compare_dynamic_tree, compare_static_tree, oracle_draft_dynamic,
                    oracle_draft_static, row_close)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


class Roundings:
    E = 0.0


@contextlib.contextmanager
def four_bits():
    """The oracle's products in 4 bits (for its draft's calls only)."""
    plain, kept, seen = M.linear, {}, Roundings()

    def linear(x, w):
        if id(w) not in kept:
            kept[id(w)] = (w, mx.term(M.widen(w)))
        q = mx.quantised(x, 2)
        size = np.linalg.norm(x, axis=1)
        seen.E = max(seen.E, (np.linalg.norm(x - q, axis=1)[size > 0] / size[size > 0]).max())
        return q @ kept[id(w)][1].T
    M.linear = linear
    try:
        yield seen
    finally:
        M.linear = plain


def models(wl, fc="random"):
    w = synth.make_target_weights(wl.dims, wl.seed)
    dr = synth.make_draft_weights(wl.dims, w, wl.seed, fc)
    return w, dr, O.Models(wl.dims, w, dr)


def engine(wl, w, dr, **kw):
    from paper_2505_14260_amd.msd import Engine
    kw = {"max_batch": 1, "max_seq": 256, "max_tree": 64, "max_prompt": 128, **kw}
    return Engine(wl.dims, w, dr, **kw)


def spec_of(paths):
    from paper_2505_14260_amd.msd import make_static_spec
    parent, rank, _ = synth.static_tree_arrays(paths)
    return make_static_spec(parent[1:], rank[1:])


def cache_rows(view, n, transposed, b=0):
    a = view[0, b, :, :, :n] if transposed else view[0, b, :, :n, :].transpose(1, 2)
    bits = a.cpu().numpy().astype(np.int16).view(np.uint16)   # [KV, hd, n]
    return M.widen(bits).transpose(2, 0, 1).reshape(n, -1)


def draft_close(eng, st, n, E, exact):
    """The draft cache's rows: `exact` marks those whose inputs are."""
    assert 0 < E < 0.0575   # of the oracle alone: below half of one term's 11.5%
    _, _, dk, dv = eng.kv_views()
    torch.cuda.synchronize()
    for view, ref, tr in ((dk, st.dkv.k, False), (dv, st.dkv.v, True)):
        got, ref = cache_rows(view, n, tr), ref[0, :n].reshape(n, -1)
        off = np.linalg.norm(got - ref, axis=1) / np.linalg.norm(ref, axis=1)
        assert (off <= 4 * E).all(), (tr, off.max(), E)
        if exact.any():
            ok, err = row_close(got[exact], ref[exact], 2.0 ** -7)
            assert ok, (tr, err)


def rtol(E):
    return 2 * E * 6 ** 0.5


NARROW = dataclasses.replace(TINY, dims=dataclasses.replace(
    WIDE.dims, d_model=168, n_heads=3, n_kv_heads=1, head_dim=64, ffn_dim=296, vocab=515))


@pytest.mark.parametrize("visual_input", ["embedding", "feature"])
@pytest.mark.parametrize("wl", [TINY, WIDE, NARROW], ids=["tiny", "wide", "narrow"])
def test_static_tree_and_caches(wl, visual_input):
    w, dr, m = models(wl)
    prompt = synth.make_prompt(wl)
    n = wl.prompt_len
    eng = engine(wl, w, dr, max_seq=n + 128, max_prompt=n, draft_mx=True, visual_input=visual_input)
    try:
        print(f"case: {wl.name}, {visual_input}", flush=True)
        first = eng.prefill(0, *prompt)
        st, ref, _, logits = O.prefill(m, *prompt, n + 128, visual_input=visual_input)
        assert argmax_ok(first, logits[-1])
        st.root = first
        if first != ref:
            st.pending[-1].e_next = m.embed(first)
        with four_bits() as seen:
            tree, logs, rank = oracle_draft_static(m, st, wl.tree.paths)
        exact = prompt[1].astype(bool) & (visual_input == "embedding")
        draft_close(eng, st, n, seen.E, exact)
        spec, trees = spec_of(wl.tree.paths), eng.new_trees(1)
        eng.draft_tree([0], spec, trees)
        got = eng.trees_to_host(trees, 1)[0]
        assert compare_static_tree(got, tree, logs, rank, rtol(seen.E)) > 0
        eng.verify([0], trees, spec.n_nodes + 1)
    finally:
        eng.close()


def test_dynamic_tree():
    from paper_2505_14260_amd.msd import make_dynamic_spec
    w, dr, m = models(TINY)
    prompt = synth.make_prompt(TINY)
    eng = engine(TINY, w, dr, draft_mx=True)
    try:
        first = eng.prefill(0, *prompt)
        st, ref, _, _ = O.prefill(m, *prompt, 256)
        assert first == ref
        K, D, N = 4, 4, 20
        with four_bits() as seen:
            tree, pool, rows, root = oracle_draft_dynamic(m, st, K, D, N)
        trees = eng.new_trees(1)
        eng.draft_tree([0], make_dynamic_spec(K, D, N), trees)
        got = eng.trees_to_host(trees, 1)[0]
        same, scored = compare_dynamic_tree(got, pool, rows, root, K, N, rtol(seen.E), ref=tree)
        assert same and scored
    finally:
        eng.close()


def test_prompt_of_several_launches():
    """2,080 rows: the products' results go through their buffer in two parts."""
    wl = dataclasses.replace(TINY, dims=dataclasses.replace(TINY.dims, n_layers=1))
    w, dr, m = models(wl)
    n = 2080
    rng = np.random.default_rng(5)
    tokens = rng.integers(0, wl.dims.vocab, n).astype(np.int32)
    vis = np.zeros(n, dtype=np.uint8)
    vis[100:1200] = 1
    rows = w["embed"][rng.integers(0, wl.dims.vocab, 1100)].copy()
    eng = engine(wl, w, dr, max_seq=n + 96, max_prompt=n, draft_mx=True)
    try:
        first = eng.prefill(0, tokens, vis, rows)
        st, ref, _, logits = O.prefill(m, tokens, vis, rows, n + 96)
        assert argmax_ok(first, logits[-1])
        if first != ref:
            st.root, st.pending[-1].e_next = first, m.embed(first)
        with four_bits() as seen:
            O.draft_catch_up(m, st)
        draft_close(eng, st, n, seen.E, vis.astype(bool))
    finally:
        eng.close()


@pytest.mark.parametrize("wl", [TINY, WIDE, NARROW], ids=["tiny", "wide", "narrow"])
def test_imported_feature(wl):
    """msd_set_state's bfloat16 feature: f_down's rounded input is exact."""
    w, dr, m = models(wl)
    d = wl.dims.d_model
    eng = engine(wl, w, dr, draft_mx=True)
    try:
        L, token = 40, 17
        rng = np.random.default_rng(d)
        h = torch.from_numpy(rng.standard_normal((1, d))).bfloat16()
        from paper_2505_14260_amd import msd
        hd = h.cuda()
        msd.msd_set_state(eng.ctx, 0, L, hd.data_ptr(), token)
        st = O.SeqState(M.KVCache(wl.dims.n_layers, 64, wl.dims.n_kv_heads, wl.dims.head_dim),
                        M.KVCache(1, 64, wl.dims.n_kv_heads, wl.dims.head_dim), L, token,
                        [O.PendingRow(False, h=h[0].double().numpy(), e_next=m.embed(token))])
        spec, trees = spec_of(["0", "1"]), eng.new_trees(1)
        eng.draft_tree([0], spec, trees)
        with four_bits() as seen:
            tree, logs, rank = oracle_draft_static(m, st, ["0", "1"])
        _, _, dk, dv = eng.kv_views()
        torch.cuda.synchronize()
        for view, ref, tr in ((dk, st.dkv.k, False), (dv, st.dkv.v, True)):
            ok, err = row_close(cache_rows(view, L, tr)[L - 1], ref[0, L - 1].reshape(-1), 2.0 ** -7)
            assert ok, (tr, err)
        assert compare_static_tree(eng.trees_to_host(trees, 1)[0], tree, logs, rank, rtol(seen.E)) > 0
    finally:
        eng.close()


@pytest.mark.parametrize("fc", ["hidden", "random"])
def test_what_is_emitted_does_not_change(fc):
    """Greedy decoding with a 4-bit draft emits the target's own tokens."""
    w, dr, m = models(TINY, fc)
    prompt = synth.make_prompt(TINY)
    eng = engine(TINY, w, dr, draft_mx=True)
    try:
        toks, cycles = eng.generate(0, prompt, spec_of(TINY.tree.paths), 48)
        ref, rows = O.greedy_generate(m, prompt, 48, return_logits=True)
        for i in range(48):
            if toks[i] != ref[i]:
                assert argmax_ok(toks[i], rows[i])
                break
        assert len(cycles) < 47 or fc == "random"   # the pass-through f_down accepts some
    finally:
        eng.close()


def decode_state(eng, prompt, cycles=3, seq=0):
    """Trees, tokens and draft caches of a few cycles."""
    spec = spec_of(TINY.tree.paths)
    T = spec.n_nodes + 1
    out = [eng.prefill(seq, *prompt)]
    trees = eng.new_trees(1)
    for _ in range(cycles):
        eng.draft_tree([seq], spec, trees)
        raw = trees.clone()
        amax, _ = eng.verify([seq], trees, T)
        em, _ = eng.accept([seq], trees, T, amax)
        out += [raw.cpu(), em]
    _, _, dk, dv = eng.kv_views()
    return out + [dk[:, seq].clone().cpu(), dv[:, seq].clone().cpu()]


def equal(a, b):
    return all(torch.equal(x, y) if torch.is_tensor(x) else x == y for x, y in zip(a, b))


def test_switching_and_repeats():
    w, dr, _ = models(TINY)
    prompt = synth.make_prompt(TINY)
    eng, plain = engine(TINY, w, dr, max_batch=2), engine(TINY, w, dr, max_batch=2)
    try:
        bf16 = decode_state(plain, prompt)
        assert equal(decode_state(eng, prompt), bf16)
        eng.use_draft_mx()
        four = decode_state(eng, prompt)
        assert not torch.equal(four[-2], bf16[-2])
        assert equal(decode_state(eng, prompt), four)
        # the other slot, in a batch with this one
        assert equal(decode_state(eng, prompt, seq=1), four)
        eng.use_draft_mx(False)
        assert equal(decode_state(eng, prompt), bf16)
        eng.use_draft_mx()
        assert equal(decode_state(eng, prompt), four)
    finally:
        eng.close()
        plain.close()


def test_ragged_batch():
    """Two sequences of different length in one tree call give what each gives alone."""
    w, dr, _ = models(TINY)
    tokens, vis, rows = synth.make_prompt(TINY)
    eng = engine(TINY, w, dr, max_batch=2, draft_mx=True)
    spec = spec_of(TINY.tree.paths)
    try:
        # a shorter prompt: the last twelve rows, text
        eng.prefill(0, tokens, vis, rows)
        eng.prefill(1, tokens[-12:], vis[-12:], None)
        both = eng.new_trees(2)
        eng.draft_tree([0, 1], spec, both)
        got = eng.trees_to_host(both, 2)
        eng.prefill(0, tokens, vis, rows)
        eng.prefill(1, tokens[-12:], vis[-12:], None)
        for b in (0, 1):
            one = eng.new_trees(1)
            eng.draft_tree([b], spec, one)
            assert bytes(eng.trees_to_host(one, 1)[0]) == bytes(got[b])
    finally:
        eng.close()


def test_an_update_reaches_the_four_bit_draft():
    w, dr, _ = models(TINY)
    prompt = synth.make_prompt(TINY)
    a, b = engine(TINY, w, dr, draft_mx=True), engine(TINY, w, dr)
    try:
        before = decode_state(a, prompt)
        for eng in (a, b):
            eng.train_accumulate(0, *prompt)
            eng.train_apply(1e-2)
        after = decode_state(a, prompt)
        b.use_draft_mx()
        assert equal(decode_state(b, prompt), after)
        assert not torch.equal(after[-2], before[-2])
    finally:
        a.close()
        b.close()


def test_refusals():
    from paper_2505_14260_amd import msd
    w, dr, _ = models(TINY)
    eng = engine(TINY, w, dr)
    small = dataclasses.replace(TINY, dims=dataclasses.replace(
        TINY.dims, n_layers=1, d_model=32, n_heads=1, n_kv_heads=1, ffn_dim=64, vocab=64))
    ws, drs, _ = models(small)
    tiny = engine(small, ws, drs)
    buf = torch.empty(msd.msd_draft_mx_bytes(eng.desc) + 512, dtype=torch.uint8, device="cuda")
    try:
        for ctx, ptr in ((None, buf.data_ptr()), (eng.ctx, buf.data_ptr() + 16),
                         (tiny.ctx, buf.data_ptr())):
            with pytest.raises(msd.MSDError) as e:
                msd.msd_set_draft_mx(ctx, ptr)
            assert e.value.code == msd.MSD_ERR_INVALID_ARG
    finally:
        eng.close()
        tiny.close()
