"""The stream on which the engine allocates its 4-bit draft weights, with stand-ins
for torch and the library's call (no GPU): torch's allocator may hand a block to the
stream current at the allocation while earlier work of that stream still uses it, so
a buffer that the engine's stream fills has to be allocated on the engine's stream."""
import contextlib
import types

import pytest

from paper_2505_14260_amd import msd


class Torch:
    """As much of torch as the call uses; notes the stream of each allocation."""
    uint8 = "uint8"

    def __init__(self):
        self.current, self.allocated = "caller's", []
        self.cuda = types.SimpleNamespace(stream=self.stream)

    @contextlib.contextmanager
    def stream(self, s):
        before, self.current = self.current, s
        try:
            yield
        finally:
            self.current = before

    def empty(self, n, dtype, device):
        self.allocated.append((n, dtype, device, self.current))
        return types.SimpleNamespace(data_ptr=lambda: 4096)


def test_the_four_bit_weights_are_allocated_on_the_engines_stream(monkeypatch):
    given = []
    monkeypatch.setattr(msd, "msd_draft_mx_bytes", lambda desc: 768)
    monkeypatch.setattr(msd, "msd_set_draft_mx", lambda ctx, ptr: given.append((ctx, ptr)))
    eng = msd.Engine.__new__(msd.Engine)
    eng.torch, eng.ctx, eng.desc, eng.dev, eng.draft_mx = Torch(), None, None, "cuda:0", None
    eng.torch_stream = "engine's"
    eng.use_draft_mx()
    assert eng.torch.allocated == [(768, "uint8", "cuda:0", "engine's")]
    assert eng.torch.current == "caller's"
    eng.use_draft_mx(False)
    eng.use_draft_mx()          # the same buffer again
    assert len(eng.torch.allocated) == 1 and given == [(None, 4096), (None, None), (None, 4096)]


@pytest.mark.gpu
def test_a_block_of_another_stream_is_not_taken():
    """Inside another stream, whose freed block of the same size is at hand."""
    torch = pytest.importorskip("torch")
    import synth
    from synth.configs import TINY
    w = synth.make_target_weights(TINY.dims, TINY.seed)
    dr = synth.make_draft_weights(TINY.dims, w, TINY.seed, "random")
    eng = msd.Engine(TINY.dims, w, dr, max_batch=1, max_seq=256, max_tree=64, max_prompt=128)
    try:
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            block = torch.empty(msd.msd_draft_mx_bytes(eng.desc), dtype=torch.uint8, device="cuda")
            address = block.data_ptr()
            del block
            eng.use_draft_mx()
        assert eng.draft_mx.data_ptr() != address
        torch.cuda.synchronize()
    finally:
        eng.close()
