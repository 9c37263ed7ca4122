"""The product's tile kernels where their loop goes round: rows of several chunks of 256 columns to a part, with parts that end before the others."""
import shutil

import pytest
import torch

from paper_2602_04163_amd import binding as bq
from test_gpu_serving import _layer, _on, dev  # noqa: F401
from test_linear_plan import plan  # noqa: F401

# n_tok and d_out for which the rule takes a tile, at every width below; with one word more to a row too
TILES = {"128x64": (129, 8200), "128x128": (65, 16400), "256x128": (129, 16400), "256x256": (515, 16400)}
WIDTHS = {1280: 256, 2304: 64, 3584: 128, 3712: 32, 3616: 32}          # columns and group: by 16 bytes but for the last


@pytest.mark.skipif(shutil.which("g++") is None, reason="no g++")
def test_the_sizes_reach_each_kernel(plan):  # noqa: F811
    for d_in in WIDTHS:
        assert [k for k, _ in plan([(n, d_in, d_out) for n, d_out in TILES.values()])] == list(TILES)
        # of f pairs of rows the gated product's tiles take 16 rows for every eight
        assert [k for k, _ in plan([(n, d_in, -(-(d_out // 2) // 8) * 16) for n, d_out in TILES.values()])] == list(TILES)


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(TILES))
@pytest.mark.parametrize("d_in", list(WIDTHS))
@pytest.mark.parametrize("bits", [1, 2, 3, 4])
def test_every_column_is_the_dequantized_one(dev, name, d_in, bits):  # noqa: F811
    """Tokens that are unit vectors give columns of What, rounded to fp16: all of them, over as many calls as that takes."""
    n, d_out = TILES[name]
    group = WIDTHS[d_in]
    print(f"chunks {name} {n} x {d_in} -> {d_out} k={bits} g={group}", flush=True)
    p, c = _on(*_layer(d_out, d_in, bits, group, d_in + bits), dev)
    want = bq.bpdq_dequant_fp16(p, c, group).t().half()
    rows = torch.arange(n, device=dev)
    for first in range(0, d_in, n):
        col = (first + rows) % d_in
        x = torch.zeros((n, d_in), dtype=torch.float16, device=dev)
        x[rows, col] = 1
        y = bq.bpdq_linear(p, c, group, x)
        assert torch.equal(y, want[col]), (first, (y != want[col]).nonzero()[:4].tolist())


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(TILES))
@pytest.mark.parametrize("d_in", [2304, 3712, 3616])
@pytest.mark.parametrize("bits", [1, 2, 3, 4])
def test_every_column_of_the_gated_product(dev, name, d_in, bits):  # noqa: F811
    """A gate that is its bias, 1, leaves the other projection's columns; an up that is 1 leaves the gate's."""
    n, d_out = TILES[name]
    group, f = WIDTHS[d_in], d_out // 2
    print(f"gated chunks {name} {n} x {d_in} -> 2 x {f} k={bits} g={group}", flush=True)
    planes, coefs = _layer(2 * f, d_in, bits, group, d_in + bits)
    coefs[:, :f] = 0
    p, c = _on(planes, coefs, dev)
    bias = torch.zeros(2 * f, dtype=torch.float16, device=dev)
    bias[:f] = 1
    want = bq.bpdq_dequant_fp16(p, c, group)[f:].t().half()
    p2, c2, bias2 = (torch.roll(t, f, axis).contiguous() for t, axis in ((p, 1), (c, 1), (bias, 0)))
    rows = torch.arange(n, device=dev)
    for first in range(0, d_in, n):
        col = (first + rows) % d_in
        x = torch.zeros((n, d_in), dtype=torch.float16, device=dev)
        x[rows, col] = 1
        y = bq.bpdq_gated_linear(p, c, group, x, bias=bias, act="none")
        assert torch.equal(y, want[col]), (first, (y != want[col]).nonzero()[:4].tolist())
        assert torch.equal(bq.bpdq_gated_linear(p2, c2, group, x, bias=bias2, act="none"), y)
