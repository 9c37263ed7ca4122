"""The product on the GPU where its kernels differ: sizes for each of them, and infinities."""
import numpy as np
import pytest
import torch

from paper_2602_04163_amd import binding as bq
from test_gpu_serving import TYPES, _layer, _on, dev  # noqa: F401

pytestmark = pytest.mark.gpu

# n_tok, d_in, d_out for which the rule takes a kernel
ROWS = {"one token": (1, 256, 130), "16 tokens": (16, 256, 520), "twice 16 tokens": (700, 256, 520)}
TILES = {"128x64": (65, 256, 8200), "128x128": (65, 256, 16400), "256x128": (129, 256, 16400), "256x256": (515, 256, 16400)}


@pytest.mark.parametrize("name", [*ROWS, *TILES])
@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_an_infinity_keeps_its_sign(dev, name, kind):  # noqa: F811
    """One infinite value under weights that are all positive makes its row's results that infinity, wherever in the columns it stands."""
    n, d_in, d_out = (ROWS | TILES)[name]
    print(f"infinities {name} {kind}", flush=True)
    planes, coefs = _layer(d_out, d_in, 2, 32, 3)
    p, c = _on(planes, np.abs(coefs) + np.float16(0.01), dev)
    x = torch.randn((n, d_in), generator=torch.Generator().manual_seed(1)).to(TYPES[kind]).to(dev)
    clean = bq.bpdq_linear(p, c, 32, x)
    for col in (0, 31, 63, 100, 127, 160, 223, 224, 255):
        for value in (float("inf"), -float("inf")):
            bad = x.clone()
            bad[n // 2, col] = value
            y = bq.bpdq_linear(p, c, 32, bad)
            assert (y[n // 2] == value).all(), (col, value, int(torch.isnan(y[n // 2]).sum()))
            y[n // 2] = clean[n // 2]
            assert torch.equal(y, clean)
