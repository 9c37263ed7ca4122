"""The norm at the ends of its range, on the GPU against the numpy oracle in 64 bits, with the tolerances of
tests/test_gpu_decoder.py."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as do
from paper_2602_04163_amd import binding as bq
from test_gpu_decoder import E, INF, NAN, TYPES, _check_norm, _norm_inputs, _np, dev  # noqa: F401

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


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,group", [(640, 64), (640, 0), (4096, 256), (4096, 0), (18944, 128), (18944, 0)])
def test_codes_of_what_is_no_number(dev, kind, d, group):  # noqa: F811
    """A group whose weight has a NaN or an infinity, and one whose values leave fp32, have no scale; the others do not see it."""
    x, _, w = _norm_inputs(3, d, kind, None, d, dev)
    per = group or d
    # (a finite weight that takes the value out of fp32: in the types that have its range)
    for value in (NAN, INF, -INF) + ((3e38,) if kind != "f16" else ()):
        for at in (3, d // 2 + 9, d - 1):
            v = w.clone()
            v[at] = value
            x2 = x.clone()
            x2[:, at] = x.abs().amax(1) + 2                # above the row's root mean square
            _, got, _ = bq.bpdq_rms_norm_q8(x2, v, group=group)
            y, _ = bq.bpdq_rms_norm(x2.float(), v.float())
            bad = ~y.isfinite().view(3, -1, per).all(2)
            assert bad[:, at // per].all() and bad.sum() == 3
            assert torch.equal(got.isnan(), bad), (value, at)
            assert got[~bad].isfinite().all()
