"""The gated product's tile kernels are the product's with other rows: what tests/test_lds_dma_linear.py checks in the assembly of those, in theirs; and the
sizes that the GPU tests give for a kernel are sizes for which it is taken."""
import os
import shutil

import pytest

import test_lds_dma_linear as product
from paper_2602_04163_amd import build
from test_lds_dma_linear import (test_a_barrier_has_its_wait_for_requests, test_a_barrier_waits_for_all_but_the_stages_ahead,  # noqa: F401
                                 test_m0_is_a_wait_state_old, test_no_lds_read_is_in_flight_at_a_barrier)
from test_linear_plan import plan  # noqa: F401

SOURCES = ["gated_k1.hip", "gated_k2.hip", "gated_k3.hip", "gated_k4.hip"]
needs_hipcc = pytest.mark.skipif(shutil.which(os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")) is None, reason="no hipcc")


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    before, product.SOURCES = product.SOURCES, SOURCES
    try:
        return product.assembly.__wrapped__(tmp_path_factory)
    finally:
        product.SOURCES = before


@pytest.fixture(params=SOURCES)
def kernels(request, assembly):
    found = assembly[request.param]
    assert len(found) == 32 and all("linear_tiles_kernel" in name for name in found)
    return found


@pytest.mark.skipif(shutil.which("g++") is None, reason="no g++")
def test_the_sizes_of_the_tests_reach_each_kernel(plan):  # noqa: F811
    """Tiles take pairs of rows by eights: of f pairs, 16 rows for every eight."""
    wanted = {(1, 256, 1000): ("rows", 1), (513, 256, 65): ("rows", 2), (257, 256, 260): ("rows", 3), (65, 256, 1550): ("rows", 5), (65, 256, 2050): ("rows", 8),
              (1500, 256, 65): ("rows x 2", 2), (700, 256, 260): ("rows x 2", 3), (513, 256, 500): ("rows x 2", 5), (257, 1024, 2500): ("128x64", 0),
              (300, 512, 4100): ("128x128", 0), (1025, 256, 2500): ("256x128", 0), (1025, 256, 4099): ("256x256", 0)}
    assert plan([(n, d_in, -(-f // 8) * 16) for n, d_in, f in wanted]) == list(wanted.values())
    here = os.path.join(os.path.dirname(os.path.abspath(__file__)), "test_gpu_decoder.py")
    assert all(f"({n}, {d_in}, {f})" in open(here).read() for n, d_in, f in wanted)


def test_every_unit_is_built():
    assert set(SOURCES) | {"gated_token.hip", "norm.hip", "rotary.hip", "sample.hip"} <= set(build.SOURCES)
