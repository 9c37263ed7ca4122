"""The product on the GPU where its kernels differ: sizes for each of them (held to the rule that chooses by tests/test_linear_plan.py),
infinities, activations, strides, alignment and magnitudes."""
import numpy as np
import pytest
import torch
from scipy.special import erfc

from oracle import serving_oracle as so
from paper_2602_04163_amd import binding as bq
from test_gpu_serving import E, TYPES, U, W16, _check_linear, _layer, _np, _on, dev  # noqa: F401

pytestmark = pytest.mark.gpu

# n_tok, d_in, d_out for which the rule takes a kernel; with one word more to a row too
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


@pytest.mark.parametrize("name", list(TILES))
@pytest.mark.parametrize("word,pad,shift", [(0, 8, 0), (0, 8, 8), (0, 5, 3), (32, 16, 8), (32, 1, 1)])
def test_tiles_of_strided_rows(dev, name, word, pad, shift):  # noqa: F811
    """Rows of X, of the residual and of Y with gaps, off 16 bytes or not, with NaN between X's rows and whatever in the workspace; Y over the
    residual; nothing but Y's rows is written; planes off 16 bytes give the same."""
    n, d_in, d_out = TILES[name]
    d_in, bits, group, t = d_in + word, 2, 32, torch.bfloat16
    print(f"tiles strided {name} d_in={d_in} pad={pad} shift={shift}", flush=True)
    planes, coefs = _layer(d_out, d_in, bits, group, n)
    g = torch.Generator().manual_seed(n)
    flat = torch.full(((n + 1) * (d_in + pad) + shift,), float("nan"), dtype=t)
    X = flat[shift:shift + n * (d_in + pad)].view(n, d_in + pad)[:, :d_in]
    X.copy_(torch.randn((n, d_in), generator=g))
    store = torch.full((n * (d_out + pad) + shift,), 7.0, dtype=t)
    rows = store[shift:].view(n, d_out + pad)
    rows[:, :d_out] = (4 * torch.randn((n, d_out), generator=g)).to(t)
    want, size = so.linear(planes, coefs, group, _np(X), None, "silu", _np(rows[:, :d_out]))
    p, c = _on(planes, coefs, dev)
    fd, sd = flat.to(dev), store.to(dev)
    Xd = fd[shift:shift + n * (d_in + pad)].view(n, d_in + pad)[:, :d_in]
    rd = sd[shift:].view(n, d_out + pad)
    Y = rd[:, :d_out]
    ws = torch.full((bq.bpdq_linear_workspace_bytes(n, d_in),), 255, dtype=torch.uint8, device=dev)
    bq.bpdq_linear(p, c, group, Xd, act="silu", residual=Y, Y=Y, ws=ws)
    _check_linear(Y, want, size, "bf16", d_in, _np(rows[:, :d_out]))
    assert (rd[:, d_out:] == 7.0).all() and (sd[:shift] == 7.0).all()
    shifted = torch.empty(p.numel() + 1, dtype=torch.int32, device=dev)
    shifted[1:] = p.flatten()
    assert torch.equal(bq.bpdq_linear(shifted[1:].view(p.shape), c, group, Xd, act="silu"), bq.bpdq_linear(p, c, group, Xd, act="silu"))


@pytest.mark.parametrize("name", list(TILES))
@pytest.mark.parametrize("word", [0, 32])
def test_tiles_of_tokens_of_all_sizes(dev, name, word):  # noqa: F811
    """bfloat16 reaches far beyond float16: tokens from 2^-120 to 2^100, each as exact as it would be alone; zeros and denormals."""
    n, d_in, d_out = TILES[name]
    d_in, group = d_in + word, 96 if word else 64
    planes, coefs = _layer(d_out, d_in, 2, group, n)
    g = torch.Generator().manual_seed(n)
    x = torch.randn((n, d_in), generator=g) * torch.exp(torch.randn(d_in, generator=g))
    x = (x * torch.exp2(torch.linspace(-120, 100, n).round())[:, None]).bfloat16()
    x[1] = 0
    x[2] = 1e-39 * torch.randn(d_in, generator=g)
    want, size = so.linear(planes, coefs, group, _np(x))
    y = _np(bq.bpdq_linear(*_on(planes, coefs, dev), group, x.to(dev)))
    # a value below 2^-29 of its token's largest is off by as much at most, times a level (below 0.3) and the columns
    tol = (W16 + (d_in + 16) * E) * size + U["bf16"] * np.abs(want) + 2.0 ** -29 * np.abs(_np(x)).max(1, keepdims=True) * d_in * 0.3 + 1e-40
    assert (np.abs(y - want) <= tol).all(), np.max(np.abs(y - want) / tol)


@pytest.mark.parametrize("name", list(TILES))
@pytest.mark.parametrize("bits", [1, 2, 3, 4])
def test_tiles_are_the_dequantized_product(dev, name, bits):  # noqa: F811
    """Tokens that are unit vectors give columns of What, rounded to fp16 and then to the type."""
    n, d_in, d_out = TILES[name]
    p, c = _on(*_layer(d_out, d_in, bits, 64, 9), dev)
    col = (37 * torch.arange(n, device=dev) + 5) % d_in
    want = bq.bpdq_dequant_fp16(p, c, 64).t()[col].half()
    for t in (torch.float16, torch.bfloat16):
        x = torch.zeros((n, d_in), dtype=t, device=dev)
        x[torch.arange(n, device=dev), col] = 1
        assert torch.equal(bq.bpdq_linear(p, c, 64, x), want.to(t))


@pytest.mark.parametrize("name", list(TILES))
@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_tiles_keep_a_nan_in_its_row(dev, name, kind):  # noqa: F811
    n, d_in, d_out = TILES[name]
    p, c = _on(*_layer(d_out, d_in, 3, 32, 5), dev)
    x = torch.randn((n, d_in), generator=torch.Generator().manual_seed(1)).to(TYPES[kind]).to(dev)
    clean = bq.bpdq_linear(p, c, 32, x)
    for row in (0, n // 2, n - 1):
        bad = x.clone()
        bad[row, 77] = float("nan")
        y = bq.bpdq_linear(p, c, 32, bad)
        assert torch.isnan(y[row]).all()
        y[row] = clean[row]
        assert torch.equal(y, clean)
