"""What stays of rows in which a mask of the type's lowest value takes part in a choice by
top_k: rows of nothing else, whose tokens all weigh alike, and rows whose temperature lets
them weigh.  Every row is compared: no top_p below falls on a whole number of tokens."""
import pytest

from test_gpu_logits import LAYOUTS, TYPES, check_choice, gen

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

HOWS = [dict(top_k=400, top_p=0.77731), dict(top_k=257, top_p=0.3331, min_p=0.5),
        dict(top_k=400, top_p=0.77731, temperature=1e45), dict(top_k=400), dict(top_k=200, top_p=0.77731),
        dict(top_p=0.77731)]


def lowest_rows(cols, type_, seed):
    """Rows of the lowest value, with 0, 3 and 300 other tokens, and of -inf with 600 of the lowest."""
    low, g = torch.finfo(TYPES[type_]).min, gen(seed)
    x = torch.full((4, cols), low)
    for r, live in ((1, 3), (2, 300)):
        x[r, torch.randperm(cols, generator=g)[:live]] = torch.randn(live, generator=g) * 2
    x[3] = float("-inf")
    x[3, torch.randperm(cols, generator=g)[:600]] = low
    return x.to(TYPES[type_])


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("how", HOWS, ids=str)
def test_top_k_among_tokens_of_the_lowest_value(how, type_):
    for n, cols in enumerate((700, 5000, 40000, 152064)):
        print(f"case: 4 x {cols} {type_}, {how}", flush=True)
        x = lowest_rows(cols, type_, n)
        assert check_choice(x, torch.rand(4, generator=gen(n)), how, LAYOUTS[n % 3]) == 0
