"""The draft in 4 bits at the width of the 7B-shaped models, where its products run on
the kernels that decoding uses (tests/test_gpu_draft_mx.py's models are narrower), against
the float64 oracle with the same roundings.  Tolerances as there."""
import dataclasses

import numpy as np
import pytest

from synth.configs import TINY, WORKLOADS
from oracle import model as M
from oracle import msd as O
from oracle import mx
from parity import compare_static_tree, oracle_draft_static, row_close
from test_gpu_draft_mx import cache_rows, engine, four_bits, models, rtol, spec_of

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_a_tree_at_full_width(monkeypatch):
    """An imported feature and a tree of three rounds; one target layer, which the draft
    phase does not read, and a quarter of the vocabulary."""
    seven = WORKLOADS["llava-1.5-7b-shaped"].dims
    wl = dataclasses.replace(TINY, dims=dataclasses.replace(seven, n_layers=1, vocab=8003))
    w, dr, m = models(wl)
    d = wl.dims.d_model
    paths = ["0", "1", "2", "3", "00", "01", "10", "11", "20", "000", "001", "100"]
    eng = engine(wl, w, dr, draft_mx=True)
    try:
        from paper_2505_14260_amd import msd
        L, token = 40, 17
        rng = np.random.default_rng(d)
        h = torch.from_numpy(rng.standard_normal((1, d))).bfloat16()
        hd = h.cuda()
        msd.msd_set_state(eng.ctx, 0, L, hd.data_ptr(), token)
        spec, trees = spec_of(paths), eng.new_trees(1)
        eng.draft_tree([0], spec, trees)
        got = eng.trees_to_host(trees, 1)[0]
        _, _, dk, dv = eng.kv_views()
        torch.cuda.synchronize()
        print("case: the oracle", flush=True)
        st = O.SeqState(M.KVCache(1, 64, wl.dims.n_kv_heads, wl.dims.head_dim),
                        M.KVCache(1, 64, wl.dims.n_kv_heads, wl.dims.head_dim), L, token,
                        [O.PendingRow(False, h=h[0].double().numpy(), e_next=m.embed(token))])
        plain = mx.term
        # row blocks: the oracle's arrays of a whole matrix would take gigabytes each
        monkeypatch.setattr(mx, "term", lambda x: np.concatenate(
            [plain(x[i:i + 256]) for i in range(0, len(x), 256)]))
        with four_bits() as seen:
            tree, logs, rank = oracle_draft_static(m, st, paths)
        for view, ref, tr in ((dk, st.dkv.k, False), (dv, st.dkv.v, True)):
            ok, err = row_close(cache_rows(view, L, tr)[L - 1], ref[0, L - 1].reshape(-1), 2.0 ** -7)
            assert ok, (tr, err)
        assert compare_static_tree(got, tree, logs, rank, rtol(seen.E)) > 0
    finally:
        eng.close()
