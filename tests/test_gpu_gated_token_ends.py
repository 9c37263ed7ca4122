"""The gated product of one token at the ends of its range, on the GPU against the numpy oracle in 64 bits, with the tolerances of
tests/test_gpu_decoder.py."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as do
from paper_2602_04163_amd import binding as bq
from test_gpu_decoder import _layer, _np, _on, dev  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d_in,group", [(256, 64), (4096, 128), (8192, 32)])
@pytest.mark.parametrize("power", [-126, -118, -100, 0, 60])
def test_gated_token_of_any_size(dev, d_in, group, power):  # noqa: F811
    """bf16 values down to the least of the type: the gate is mostly a bias that brings the result inside the type, the other projection has the
    token's size."""
    f = 50
    planes, coefs = _layer(2 * f, d_in, 2, group, d_in)
    g = torch.Generator().manual_seed(power % 1000)
    x = (torch.randn((1, d_in), generator=g, dtype=torch.float64) * 2.0 ** power).bfloat16().to(dev)
    b = torch.zeros(2 * f, dtype=torch.bfloat16, device=dev)
    p, c = _on(planes, coefs, dev)
    if power < 0:
        b[:f] = 2.0 ** (-power // 2)
    y = bq.bpdq_gated_linear(p, c, group, x, bias=b, act="none")
    want, (gate, up), (size_g, size_u), _ = do.gated(planes, coefs, group, _np(x), _np(b), "none")
    # sums of exact products in fp32: (d_in + 16) roundings of the size at most, each projection, and the result's
    e = (d_in + 16) * 2.0 ** -24
    tol = e * (size_g * np.abs(up) + size_u * np.abs(gate)) * (1 + e) + 2.0 ** -8 * np.abs(want) + 2.0 ** -133
    got = _np(y)
    assert (np.abs(got - want) <= tol).all(), np.max(np.abs(got - want) / tol)
    assert np.linalg.norm(got - want) <= (2.0 ** -8 + 2.0 ** -16) * np.linalg.norm(want) + 2.0 ** -133 * f
