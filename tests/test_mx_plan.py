"""The kernels that products are dispatched to, from the plan itself (no GPU): the GPU
tests' products reach every one of them, so that another fit of the plan cannot take a
kernel out of the tests unseen."""
import os
import shutil
import subprocess

import pytest

pytest.importorskip("torch")

from test_gpu_mx_kernels import PRODUCTS  # noqa: E402

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2505_14260_amd", "csrc")
MAIN = r"""
#include "mx_plan.h"
#include <cstdio>
int main() {
  int M, N, K, terms;
  while (scanf("%d %d %d %d", &M, &N, &K, &terms) == 4) {
    const msd::ProductPlan p = msd::plan_product(M, N, (K + msd::MX_GROUP - 1) / msd::MX_GROUP, terms);
    printf("%d %d %d %d\n", p.MT, p.CT, p.BM, p.BN);
  }
}
"""

# (16-row tiles, 16-column tiles) of the split kernel, (rows, columns) of the tile kernel
KERNELS = [("split", m, c) for m in (1, 2, 4) for c in (1, 2, 4)] + \
          [("tile", 64, 128), ("tile", 128, 256), ("tile", 256, 256)]


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(MAIN)
    exe = str(d / "plan")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-I", CSRC, "-o", exe, str(d / "plan.cpp")])

    def kernels(products):
        """(kernel, ..) of each (rows, columns, length, terms)."""
        text = "".join("%d %d %d %d\n" % p for p in products)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
        plans = [tuple(map(int, line.split())) for line in out.splitlines()]
        assert len(plans) == len(products)
        return [("split", m, c) if c else ("tile", bm, bn) for m, c, bm, bn in plans]
    return kernels


@pytest.mark.parametrize("terms", [1, 2])
def test_the_gpu_tests_reach_every_kernel(plan, terms):
    products = [(r, n, k, terms) for (n, k), rows in PRODUCTS.items() for r in rows]
    run = {}
    for p, kernel in zip(products, plan(products)):
        run.setdefault(kernel, []).append(p)
    assert set(run) == set(KERNELS)
    for (kind, a, b), ps in run.items():
        high, wide = (16 * a, 16 * b) if kind == "split" else (a, b)
        # a last tile of rows and one of columns that are cut
        assert any(r % high for r, _, _, _ in ps), (kind, a, b)
        assert any(n % wide for _, n, _, _ in ps), (kind, a, b)
    # of one workgroup and of several along the rows; of fewer rows than a tile
    assert any(r < 64 for r, _, _, _ in run["tile", 64, 128])
    assert any(r > 64 for r, _, _, _ in run["tile", 64, 128])
    # eight waves share K's groups of 512 columns: a group a wave, and a second one
    for c in (1, 2, 4):
        at = [p for m in (1, 2, 4) for p in run["split", m, c]]
        assert {-(-k // 512) > 8 for _, _, k, _ in at} == {False, True}, c


def test_the_plan_takes_any_size(plan):
    """The ends of the operators' ranges, and rows that change the kernel."""
    sizes = [(1, 1, 1), (1 << 23, 1, 1), (1, 1 << 23, 1), (1, 1, 1 << 20), (2048, 1 << 15, 1 << 20),
             (16, 4096, 11008), (17, 4096, 11008)]
    got = plan([(*s, t) for s in sizes for t in (1, 2)])
    assert set(got) <= set(KERNELS)
    # the rows that a workgroup takes follow the rows that there are
    for t in (1, 2):
        for rows, tiles in ((16, 1), (17, 2), (32, 2), (33, 4)):
            assert plan([(rows, 4096, 11008, t)])[0][:2] == ("split", tiles)
