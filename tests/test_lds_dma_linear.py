"""What the tile kernels of the product leave to their source where they feed LDS by LDS-DMA, checked in the assembly that the compiler
makes of them: M0 is a wait state old when a request reads it, no LDS read is in flight at a barrier behind which a request may
overwrite what it reads, and every barrier between request and reading has its wait for requests before it."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2602_04163_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no hipcc")


SOURCES = ["linear_k1.hip", "linear_k2.hip", "linear_k3.hip", "linear_k4.hip"]


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    """source -> function -> its instructions and labels, of the kernels that request by LDS-DMA; all compiled at once"""
    folder = tmp_path_factory.mktemp("asm")
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]

    def compiled(source):
        out = folder / (source + ".s")
        subprocess.run([HIPCC, *flags, "--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o", str(out)],
                       check=True, capture_output=True)
        found = {}
        for m in re.finditer(r"^(_ZN4bpdq\w+):[^\n]*\n(.*?)^\.Lfunc_end", out.read_text(), re.S | re.M):
            ops = [op for op in (line.split(";")[0].strip() for line in m.group(2).split("\n"))
                   if op and (not op.startswith(".") or op.startswith(".LBB"))]
            if any("load_lds" in op for op in ops):
                found[m.group(1)] = ops
        return found

    with ThreadPoolExecutor(len(SOURCES)) as pool:
        return dict(zip(SOURCES, pool.map(compiled, SOURCES)))


@pytest.fixture(params=SOURCES)
def kernels(request, assembly):
    found = assembly[request.param]
    # two types, four tiles, four forms each
    assert len(found) == 32 and all("linear_tiles_kernel" in name for name in found)
    return found


def test_m0_is_a_wait_state_old(kernels):
    for name, ops in kernels.items():
        ops = [op for op in ops if not op.endswith(":")]
        for before, op in zip(ops, ops[1:]):
            assert "load_lds" not in op or not re.match(r"s_\w+ m0\b", before), name


def _after(ops):
    label = {op[:-1]: i for i, op in enumerate(ops) if op.endswith(":")}
    out = []
    for i, op in enumerate(ops):
        to = [label[op.split()[-1]]] if op.startswith(("s_cbranch", "s_branch")) else []
        if not op.startswith(("s_branch", "s_endpgm")) and i + 1 < len(ops):
            to.append(i + 1)
        out.append(to)
    return out


def test_no_lds_read_is_in_flight_at_a_barrier(kernels):
    for name, ops in kernels.items():
        after = _after(ops)
        todo, done = [j for i, op in enumerate(ops) if op.startswith("ds_read") for j in after[i]], set()
        while todo:
            i = todo.pop()
            if i in done:
                continue
            done.add(i)
            if ops[i].startswith("s_waitcnt") and "lgkmcnt(0)" in ops[i]:
                continue
            assert not ops[i].startswith("s_barrier"), name
            todo += after[i]


def test_a_barrier_has_its_wait_for_requests(kernels):
    """Between a request and the next barrier stands a wait for vector memory; in the loop it lets one stage's requests be outstanding."""
    for name, ops in kernels.items():
        after = _after(ops)
        todo, done = [j for i, op in enumerate(ops) if "load_lds" in op for j in after[i]], set()
        while todo:
            i = todo.pop()
            if i in done:
                continue
            done.add(i)
            if ops[i].startswith("s_waitcnt") and "vmcnt(" in ops[i]:
                continue
            assert not ops[i].startswith("s_barrier"), name
            todo += after[i]


def _dma(name):
    """Requests of a wavefront per stage, and stages, from the tile in a kernel's name."""
    _, wr, wt, _, _, tt, stages = map(int, re.search("LinearTileI" + r"Li(\d+)E" * 7, name).groups())
    return 32 * tt * wt * 128 // 1024 // (wr * wt), stages


def test_a_barrier_waits_for_all_but_the_stages_ahead(kernels):
    """What stands between a request and the next barrier leaves at most the requests of the stages behind the next one outstanding, and before
    the loop the first quarter of the last stage's too.  (Other vector memory operations in between make a wait longer, not shorter.)"""
    for name, ops in kernels.items():
        per_stage, stages = _dma(name)
        after = _after(ops)

        def walk(limit):
            """Barriers that a request reaches without a wait for all but `limit` in between."""
            todo, done, reached = [j for i, op in enumerate(ops) if "load_lds" in op for j in after[i]], set(), set()
            while todo:
                i = todo.pop()
                if i in done:
                    continue
                done.add(i)
                count = re.search(r"vmcnt\((\d+)\)", ops[i]) if ops[i].startswith("s_waitcnt") else None
                if count and int(count.group(1)) <= limit:
                    continue
                if ops[i].startswith("s_barrier"):
                    reached.add(i)
                    continue
                todo += after[i]
            return reached

        def repeats(i):
            todo, done = list(after[i]), set()
            while todo:
                j = todo.pop()
                if j in done:
                    continue
                done.add(j)
                todo += after[j]
            return i in done

        ahead = (stages - 2) * per_stage
        loop = [i for i, op in enumerate(ops) if op.startswith("s_barrier") and repeats(i)]
        assert loop and not walk(ahead + per_stage // 4), name
        assert not walk(ahead) & set(loop), name
