"""What the quantising operators leave in memory: codes and scales read on the host by
the layout that csrc/k_mx.hip documents, against the oracle, without the library's own
way back.

Tiles of 16 rows x 128 columns of one term, 1 KB: lane l's 16 bytes (row l % 16, block
l / 16 of four; two values a byte, the lower nibble first) at 16 l.  Per 16 rows the
tiles of term 0 in sequence, then those of term 1.  The scales of four neighbouring
tiles take 256 bytes, lane l's four at 4 l.  Columns past the last are zero, scales too;
rows past the last are zero in weights and untouched in activations.
"""
import numpy as np
import pytest

from oracle import mx as O
from test_gpu_mx import gen, matrix, strided, values, wild

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

VALUE = np.concatenate([O.GRID, -O.GRID])
CODE_FILL, SCALE_FILL = 0xF7, 0xF1   # what matrix() leaves in the buffers


def decode(q):
    """codes [terms][rows padded to 16][tiles * 128] and scales [terms][rows][groups * 16]
    (one per block of 32 columns, four tiles' worth per group) of a quantised matrix."""
    rows, cols = q.shape
    r16, nkt, ng, T = -(-rows // 16), -(-cols // 128), -(-cols // 512), q.terms
    c = q.codes.cpu().numpy().reshape(r16, T, nkt, 4, 16, 16)    # tile, block, row, byte
    c = np.stack([c & 15, c >> 4], -1).reshape(r16, T, nkt, 4, 16, 32)
    codes = c.transpose(1, 0, 4, 2, 3, 5).reshape(T, r16 * 16, nkt * 128)
    s = q.scales.cpu().numpy().reshape(r16, T, ng, 4, 16, 4)     # group, block, row, tile
    return codes, s.transpose(1, 0, 4, 2, 5, 3).reshape(T, r16 * 16, ng * 16)


def exponents(x):
    """The scale codes of a matrix's blocks, from the definition."""
    rows, cols = x.shape
    b = np.zeros((rows, -(-cols // 32) * 32))
    b[:, :cols] = np.abs(x)
    top = b.reshape(rows, -1, 32).max(-1)
    e = np.where(top > 0, np.frexp(np.where(top > 0, top, 1.0))[1] - 1 - 2, -127)
    return np.clip(e, -127, 127) + 127


def padding(q, codes, scales):
    rows, cols = q.shape
    assert not scales[:, :rows, -(-cols // 32):].any()
    # -0 stands for zero too: the lower three bits count
    assert not (codes[:, :rows, cols:] & 7).any()
    if q.layout == "weight":
        assert not codes[:, rows:].any() and not scales[:, rows:].any()
    else:
        fill = np.tile([CODE_FILL & 15, CODE_FILL >> 4], codes.shape[2] // 2)
        assert (codes[:, rows:] == fill).all() and (scales[:, rows:] == SCALE_FILL).all()


def term_values(q, codes, scales, t):
    rows, cols = q.shape
    size = np.ldexp(1.0, scales[t, :rows, :-(-cols // 32)].astype(int) - 127)
    return VALUE[codes[t, :rows, :cols]] * size.repeat(32, 1)[:, :cols]


SIZES = [(1, 1), (16, 128), (17, 129), (15, 511), (33, 513), (5, 1500), (70, 2056), (130, 640)]


@pytest.mark.parametrize("layout, terms", [("rows", 1), ("rows", 2), ("weight", 1)])
def test_quantised_rows(layout, terms):
    from paper_2505_14260_amd import mx
    for i, (rows, cols) in enumerate(SIZES):
        print(f"case: {rows} x {cols}", flush=True)
        x = wild(rows, cols, i)
        q = matrix(rows, cols, layout, terms)
        mx.quantize(strided(x, 3, 1), q)
        codes, scales = decode(q)
        padding(q, codes, scales)
        left = x.double().numpy()
        for t in range(terms):
            want = O.term(left)
            assert np.array_equal(scales[t, :rows, :-(-cols // 32)], exponents(left)), t
            assert np.array_equal(term_values(q, codes, scales, t), want), t
            left = left - want


@pytest.mark.parametrize("rows, cols", [(1, 1), (17, 129), (33, 513), (70, 2056), (129, 4100)])
def test_norm_and_swiglu(rows, cols):
    """The same layout: what the host reads is what the library's way back gives."""
    from paper_2505_14260_amd import mx
    x, y = wild(rows, cols, 1, 3).cuda(), wild(rows, cols, 2, 3).cuda()
    gain = (1 + 0.2 * torch.randn(cols, generator=gen(8))).bfloat16().cuda()
    for call in (lambda q: mx.resid_norm(x, y, gain, 1e-5, None, q), lambda q: mx.swiglu(x, y, q)):
        q = matrix(rows, cols)
        call(q)
        codes, scales = decode(q)
        padding(q, codes, scales)
        got = term_values(q, codes, scales, 0) + term_values(q, codes, scales, 1)
        assert np.array_equal(got.astype(np.float32), values(q).astype(np.float32))
