"""The words and coefficients that a wavefront of the product's tile kernels requests into LDS for itself, by LDS-DMA, checked in the assembly that the
compiler makes: planes that go by 16 bytes are requested so in every tile, and nothing is read, or requested over, ahead of a wait that covers its
request."""
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


def _reached(ops, after, start, ends):
    """Instructions for which `ends` holds that `start` reaches without a wait that covers it: one for at most as many vector memory operations as were
    issued since, on the path with the fewest."""
    vector = [re.match(r"(global|buffer|scratch|flat)_", op) is not None for op in ops]
    least, todo, found = {}, [(j, 0) for j in after[start]], set()
    while todo:
        i, since = todo.pop()
        if least.get(i, 64) <= since:
            continue
        least[i] = since
        count = re.search(r"vmcnt\((\d+)\)", ops[i]) if ops[i].startswith("s_waitcnt") else None
        if count and int(count.group(1)) <= since:
            continue
        if ends(ops[i]):
            found.add(i)
            continue
        todo += [(j, min(63, since + vector[i])) for j in after[i]]
    return found


def test_what_a_wavefront_requests_for_itself_is_waited_for(kernels):
    """Coefficients, and words by ones, are read behind a wait that covers their request.  These and words by fours are covered before the next barrier
    too, behind which a region may be requested anew or, words by fours, is read; of X, which the same instruction requests, the first stage
    alone is."""
    for name, ops in kernels.items():
        k, vec, per_stage, rt = _form(name)
        after = product._after(ops)
        requests = {kind: [i for i, op in enumerate(ops) if op.startswith(f"global_load_lds_{kind} ")] for kind in ("ushort", "dword", "dwordx4")}
        assert len(requests["ushort"]) >= 2 * rt * (k + 1), name
        for kind, read in (("ushort", r"ds_read_u16"), ("dword", r"ds_read2?(st64)?_b32")):
            for i in requests[kind]:
                assert not _reached(ops, after, i, lambda op: re.match(read, op) or op.startswith("s_barrier")), (name, ops[i])
        open_at_barrier = [i for i in requests["dwordx4"] if _reached(ops, after, i, lambda op: op.startswith("s_barrier"))]
        words = len(requests["dwordx4"]) - len(open_at_barrier) - per_stage
        assert len(open_at_barrier) == 5 * per_stage + per_stage // 4, name
        assert words in ((2 * rt * k, 5 * k) if vec else (0,)), (name, words)
