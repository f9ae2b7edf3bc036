"""A teacher's record has to be on the engine's own device: its pointers are read there.
Stand-ins for the tensors, the streams and the library's call (no GPU)."""
import contextlib
import types

import pytest

from paper_2505_14260_amd import msd

torch = pytest.importorskip("torch")


def record(device, dtype, rows=5, k=3):
    t = torch.empty(rows, k, dtype=dtype, device="meta")
    return types.SimpleNamespace(dtype=t.dtype, shape=t.shape, dim=t.dim, is_contiguous=t.is_contiguous,
                                 is_cuda=device.type == "cuda", device=device, data_ptr=lambda: 4096)


def engine():
    eng = msd.Engine.__new__(msd.Engine)
    eng.dev, eng.ctx = torch.device("cuda"), None
    eng.torch_stream = types.SimpleNamespace(device=torch.device("cuda:1"), wait_stream=lambda s: None)
    eng.torch = types.SimpleNamespace(
        int32=torch.int32, float32=torch.float32,
        cuda=types.SimpleNamespace(current_stream=lambda d: None, stream=contextlib.nullcontext))
    return eng


def test_a_record_on_another_device_is_refused(monkeypatch):
    given = []
    monkeypatch.setattr(msd, "msd_train_accumulate_top", lambda *a: given.append(a))
    here, other = torch.device("cuda:1"), torch.device("cuda:0")
    for at_ids, at_values in ((other, here), (here, other), (other, other)):
        teacher = (record(at_ids, torch.int32), record(at_values, torch.float32), 1.0)
        with pytest.raises(ValueError, match="cuda:1"):
            engine().train_accumulate(0, [1] * 6, [0] * 6, None, teacher)
    assert not given
    engine().train_accumulate(0, [1] * 6, [0] * 6, None,
                              (record(here, torch.int32), record(here, torch.float32), 1.0))
    assert len(given) == 1
