"""The norm at the ends of its range, on the GPU against the numpy oracle in 64 bits, with the tolerances of
tests/test_gpu_decoder.py."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as do
from paper_2602_04163_amd import binding as bq
from test_gpu_decoder import E, TYPES, _check_norm, _np, dev  # noqa: F401

pytestmark = pytest.mark.gpu


def _loud(n, d, kind, seed, most, dev):  # noqa: F811
    g = torch.Generator().manual_seed(seed)
    x = ((2 * torch.rand((n, d), generator=g, dtype=torch.float64) - 1) * most).to(TYPES[kind])
    return x.to(dev), (1 + 0.3 * torch.randn(d, generator=g)).to(TYPES[kind]).to(dev)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("most", [1e37, 5e37, 3e38])
def test_norm_of_the_largest_values(dev, kind, most):  # noqa: F811
    """One over the root is below fp32's normal numbers from a root of 8.5e37 on, and times a weight sooner."""
    for d in (96, 4000):
        x, w = _loud(5, d, kind, d, most, dev)
        w[::3] *= 0.01
        y, _ = bq.bpdq_rms_norm(x, w)
        want = _check_norm(y, None, x, None, w, kind, None)
        codes, scales, _ = bq.bpdq_rms_norm_q8(x, w, group=32)
        step = do.scales(want, 32)
        assert (np.abs(_np(scales) - step) <= 12 * E * step).all()
        exact = want.reshape(5, -1, 32) / step[:, :, None]
        assert (np.abs(_np(codes).reshape(exact.shape) - exact) <= 0.5 + 127 * 12 * E).all()


def test_norm_of_large_and_small_weights(dev):  # noqa: F811
    """The result is of ordinary size where the weight makes up for the root."""
    for most, by in ((1e30, 1e20), (1e-18, 1e-30), (1e30, 1e-20), (1e-18, 1e30)):
        x, w = _loud(4, 500, "f32", 3, most, dev)
        y, _ = bq.bpdq_rms_norm(x, w * by, eps=1e-37)
        _check_norm(y, None, x, None, w * by, "f32", None, eps=float(np.float32(1e-37)))
