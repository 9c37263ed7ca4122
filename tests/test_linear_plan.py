"""The rule that chooses the kernel of the product on stored planes, compiled for the host: the sizes that the GPU tests give for a kernel
are sizes for which it is taken."""
import os
import shutil
import subprocess

import pytest

from paper_2602_04163_amd import build
from test_gpu_serving_tiles import ROWS, TILES

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no g++")

MAIN = """
#include "linear_plan.h"
#include <cstdio>
#include <cstdlib>
int main(int n, char** v) {
  const char* name[] = {"rows", "rows x 2", "256x256", "256x128", "128x128", "128x64"};
  for (int i = 1; i + 2 < n; i += 3) {
    const bpdq::LinearPlan p = bpdq::linear_plan(std::atoi(v[i]), std::atoi(v[i + 1]), std::atoi(v[i + 2]));
    std::printf("%s,%d\\n", name[p.kernel], p.r);
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    folder = tmp_path_factory.mktemp("plan")
    (folder / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-I", build.CSRC, str(folder / "main.cpp"), "-o", str(folder / "main")], check=True)

    def of(sizes):
        out = subprocess.run([str(folder / "main"), *[str(v) for size in sizes for v in size]], check=True, capture_output=True, text=True)
        return [(name, int(r)) for name, r in (line.split(",") for line in out.stdout.splitlines())]
    return of


def test_the_sizes_of_the_tests_reach_each_kernel(plan):
    for d_in in (256, 288):
        assert [k for k, _ in plan([(n, d_in, d_out) for n, _, d_out in TILES.values()])] == list(TILES)
    assert [k for k, _ in plan(list(ROWS.values()))] == ["rows", "rows", "rows x 2"]


def test_the_rule(plan):
    """Up to 32 tokens no kernel takes the ordered X, for which there is no workspace; in the tile kernels offsets fit 32 bits."""
    sizes = [(n, d_in, d_out) for n in (1, 2, 16, 17, 31, 32) for d_in in (32, 4096, 18944) for d_out in (1, 100, 18944, 200000)]
    assert all(k in ("rows", "rows x 2") for k, _ in plan(sizes))
    assert all(r in ((1, 2, 3, 5, 8) if k == "rows" else (2, 3, 5)) for k, r in plan(sizes))
    assert plan([(4096, 3584, 18944), (4096, 1 << 20, 18944)]) == [("256x256", 0)] * 2
    assert plan([(4096, (1 << 20) + 32, 18944)])[0][0] in ("rows", "rows x 2")
