"""Sampling at the ends of what a weight counts, on the GPU against the numpy oracle in 64 bits, with the tolerances of
tests/test_gpu_decoder.py."""
import numpy as np
import pytest
import torch

from paper_2602_04163_amd import binding as bq
from test_gpu_decoder import E, INF, _check_sample, dev  # noqa: F401

pytestmark = pytest.mark.gpu


def _last_of(x, dev, **asked):  # noqa: F811
    """The last token that is kept (u = 1)."""
    one = {k: torch.full((x.shape[0],), v, dtype=torch.int32 if k == "top_k" else torch.float32, device=dev) for k, v in asked.items()}
    return bq.bpdq_sample(x, torch.ones(x.shape[0], device=dev), want_prob=True, **one)


@pytest.mark.parametrize("rows", [1, 300])
def test_sample_keeps_what_rounds_to_a_unit(dev, rows):  # noqa: F811
    """Weights between half a unit of 2^-43 and one count as one: the last of them is the last token, whatever bounds the row and however it is cut.
    A top-k of 300 of 4000 values is found in the histogram, with 600 values in its border's bin."""
    x = torch.full((rows, 4000), -INF)
    x[:, 5] = 0.0
    x[:, 1000:1600] = -60.0                              # no weight
    x[:, [7, 2000, 3900]] = -43.5 * float(np.log(2.0))   # 2^-43.5
    x = x.to(dev)
    for asked in (dict(top_k=300), dict(top_k=300, top_p=0.99), dict(), dict(min_p=2.0 ** -44)):
        token, prob = _last_of(x, dev, **asked)
        if "top_p" in asked:
            assert (token == 5).all() and (prob == 1).all(), asked
        else:
            assert (token == 3900).all(), (asked, token[:4])
            assert (prob == np.float32(2.0 ** -43)).all(), asked


@pytest.mark.parametrize("units", [2, 9, 100])
def test_sample_keeps_what_rounds_to_min_p(dev, units):  # noqa: F811
    """Of a min-p of so many units, weights from half a unit below it on."""
    x = torch.full((3, 4000), -INF)
    x[:, 5] = 0.0
    x[:, 1000:1600] = -60.0
    x[:, [7, 2000, 3800]] = float(np.log((units - 0.4) * 2.0 ** -43))
    x[:, 3900] = float(np.log((units - 0.6) * 2.0 ** -43))
    x = x.to(dev)
    for asked in (dict(), dict(top_k=300)):
        token, prob = _last_of(x, dev, min_p=units * 2.0 ** -43, **asked)
        assert (token == 3800).all(), (asked, token)
        assert ((prob - units * 2.0 ** -43).abs() <= 4 * E * units * 2.0 ** -43).all()


def test_sample_distances_beyond_fp32(dev):  # noqa: F811
    """Values whose difference is infinite in fp32, at temperatures at which both count."""
    x = torch.full((6, 40), -3e38, device=dev)
    x[:, [1, 20]] = 3e38
    x[:, 30] = 0.0
    u = [0.0, 0.02, 0.13, 0.4, 0.7, 0.99]
    for t in (3e38, 1e38, 3e37):
        for asked in (dict(m=[0.001] * 6), dict(k=[35] * 6), dict(k=[30] * 6, m=[0.05] * 6), dict(p=[0.9] * 6, m=[0.001] * 6)):
            _check_sample(x, u, t=[t] * 6, dev=dev, **asked)
