"""The product on the GPU where its kernels differ: sizes for each of them, infinities, activations."""
import numpy as np
import pytest
import torch
from scipy.special import erfc

from paper_2602_04163_amd import binding as bq
from test_gpu_serving import TYPES, U, _layer, _np, _on, dev  # noqa: F401

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


def _activation(v, act):
    """The activation of v in 64 bits, and the size of the exponential's argument in it."""
    if act == "gelu":
        return 0.5 * v * erfc(-v / np.sqrt(2.0)), v * v / 2
    if act == "gelu_tanh":
        u = np.sqrt(2.0 / np.pi) * (v + 0.044715 * v ** 3)
        return v / (1.0 + np.exp(-2 * u)), np.abs(2 * u)
    if act == "silu":
        return v / (1.0 + np.exp(-v)), np.abs(v)
    return (np.maximum(v, 0.0) if act == "relu" else v), 0 * v


@pytest.mark.parametrize("name", [*ROWS, *TILES])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_activations_to_the_last_bits(dev, name, act, kind):  # noqa: F811
    """act(bias), of tokens that are zero, over the range in which the results are numbers: the relative error of the activation itself is below
    2^-16 and 8 e of the exponential's argument (that many roundings are in it), and the result is rounded once."""
    n, d_in, d_out = (ROWS | TILES)[name]
    print(f"activation {name} {act} {kind}", flush=True)
    planes, coefs = _layer(d_out, d_in, 1, 256, 5)
    p, c = _on(planes, coefs, dev)
    # the ends are those of exp in fp32 for the largest argument, v^3 in gelu_tanh
    bias = torch.linspace(-9, 9, d_out, dtype=torch.float64).to(TYPES[kind])
    y = _np(bq.bpdq_linear(p, c, 256, torch.zeros((n, d_in), dtype=TYPES[kind], device=dev), bias=bias.to(dev), act=act))
    v = _np(bias)
    want, arg = _activation(v, act)
    tol = (U[kind] + (2.0 ** -16 + 8 * 2.0 ** -24 * arg) * 1.01) * np.abs(want) + (2.0 ** -25 if kind == "f16" else 2.0 ** -126)
    off = np.abs(y - want[None, :]) / tol
    assert (off <= 1).all(), (v[np.argwhere(off > 1)[:5, 1]], off.max())
