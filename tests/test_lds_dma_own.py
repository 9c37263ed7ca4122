"""The words and coefficients that a wavefront of the product's tile kernels requests into LDS for itself, by LDS-DMA, checked in the assembly that the
compiler makes: planes that go by 16 bytes are requested so in every tile."""
import re

import pytest

import test_lds_dma_linear as product
from test_lds_dma_linear import pytestmark  # noqa: F401

SOURCES = [f"{kind}_k{k}.hip" for kind in ("linear", "gated") for k in (1, 2, 3, 4)]


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    before, product.SOURCES = product.SOURCES, SOURCES
    try:
        return product.assembly.__wrapped__(tmp_path_factory)
    finally:
        product.SOURCES = before


@pytest.fixture(params=SOURCES)
def kernels(request, assembly):
    return assembly[request.param]


def _form(name):
    """Planes, whether they go by 16 bytes, requests of X to a stage, and blocks of rows, from a kernel's name."""
    k, _, _, _, rt, _, _ = map(int, re.search("LinearTileI" + r"Li(\d+)E" * 7, name).groups())
    _, vec, _ = re.search(r"Li(\d)ELb(\d)ELb(\d)EEEv", name).groups()
    return k, vec == "1", product._dma(name)[0], rt


def test_planes_that_go_by_16_bytes_are_requested_so(kernels):
    """Four words at a time: by one at a time a lane asks for 16 bytes of a line in four requests."""
    kinds = set()
    for name, ops in kernels.items():
        vec = _form(name)[1]
        kinds.add(vec)
        assert any(op.startswith("global_load_lds_dword ") for op in ops) != vec, name
    assert kinds == {False, True}
