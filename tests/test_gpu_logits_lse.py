"""The log-sum-exp that distillation writes, for rows whose loss is not a number too: of the
logits alone, NaN for a NaN or +inf among them, -inf for a row of -inf (tolerance: the header
of test_gpu_logits.py)."""
import numpy as np
import pytest

from oracle import logits as O
from test_gpu_logits import TYPES, U, f32, gen, host, record, rows_of, sum_error

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("type_", list(TYPES))
def test_log_sum_exp_of_every_kind_of_row(type_):
    from paper_2505_14260_amd import logits as L
    # (with 260 rows the kernels for more rows than compute units)
    for rows, cols in ((10, 9), (10, 3000), (10, 40000), (10, 262144), (260, 3000), (260, 32000),
                       (260, 81920)):
        print(f"case: log-sum-exp, {rows} x {cols} {type_}", flush=True)
        x = rows_of(10, cols, cols)
        ids, v = record(x, 8, 1)
        x[0] = float("-inf")
        x[1] = float("-inf")
        ids[1] = -1
        x[2, cols // 2] = float("nan")
        x[3, cols - 1] = float("inf")
        x[4] = float("nan")
        v[5, 3] = float("nan")                # the teacher's: not the logits'
        v[6] = float("-inf")
        ids[7] = cols
        x[8, : cols - 1] = float("-inf")
        x[9, :] = float("inf")
        x = x.to(TYPES[type_])
        again = torch.arange(rows) % 10
        xs, idd, vd = x[again].cuda(), ids[again].cuda(), v[again].cuda()
        alone, fused, dx = f32(rows), f32(rows), torch.empty_like(xs)
        L.distill(xs, idd, vd, 1.5, f32(rows), alone)
        L.distill(xs, idd, vd, 1.5, f32(rows), fused, torch.rand(rows, generator=gen(2)).cuda(), dx)
        for lse in (host(alone), host(fused)):
            for r in range(rows):
                want = O.distill(host(x[r % 10]), ids[r % 10].numpy(), v[r % 10].numpy(), 1.5)[1] \
                    if r < 10 else lse[r % 10]
                if np.isfinite(want):
                    tol = (sum_error(host(x[r % 10]), 1.5)[0] + U * abs(want)) if r < 10 else 0
                    assert abs(lse[r] - want) <= tol, (r, lse[r], want)
                else:
                    assert np.array_equal(lse[r], want, equal_nan=True), (r, lse[r], want)
