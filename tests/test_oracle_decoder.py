"""The oracle of the norm, rotary positions and the choice of a token, pinned against other ways to the same result."""
import itertools
import math

import numpy as np
import pytest

from oracle import decoder_oracle as do


def test_norm_has_unit_mean_square():
    g = np.random.default_rng(1)
    x, r = g.standard_normal((5, 37)), g.standard_normal((5, 37))
    s, y = do.rms_norm(x, r, eps=0.0)
    assert np.allclose(s, x + r) and np.allclose((y * y).mean(1), 1.0)
    _, z = do.rms_norm(1e3 * (x + r), weight=np.full(37, 0.25), offset=1.0, eps=0.0)
    assert np.allclose(z, 1.25 * y)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_depends_on_distances_alone(layout):
    """<R_p q, R_t k> = <R_{p - t} q, k>, lengths stay, the inverse turns back, and channels behind the turned ones are as they were."""
    g = np.random.default_rng(2)
    q, k = g.standard_normal((1, 1, 24)), g.standard_normal((1, 1, 24))
    freq, _ = do.rotary_frequencies(16, 100.0)
    turn = lambda x, p, **kw: do.rotary(x, np.array([float(p)]), freq, layout, **kw)  # noqa: E731
    for p, t in [(5, 3), (1000, 17), (40, 40)]:
        assert math.isclose((turn(q, p) * turn(k, t)).sum(), (turn(q, p - t) * k).sum(), abs_tol=1e-9)
    assert np.allclose(turn(turn(q, 9), 9, inverse=True), q)
    assert math.isclose((turn(q, 77) ** 2).sum(), (q ** 2).sum()) and (turn(q, 77)[..., 16:] == q[..., 16:]).all()


def test_frequencies():
    plain, one = do.rotary_frequencies(64)
    assert plain[0] == 1.0 and math.isclose(plain[16], 0.01) and one == 1.0
    for kind in ("yarn", "bands"):
        f, m = do.rotary_frequencies(64, scaling=kind, factor=8.0)
        ratio = plain / f
        assert ratio[0] == 1.0 and math.isclose(ratio[-1], 8.0) and (np.diff(ratio) >= -1e-12).all()
        assert m == (0.1 * math.log(8.0) + 1 if kind == "yarn" else 1.0)
    f, _ = do.rotary_frequencies(64, scaling="ntk", factor=8.0)
    assert f[0] == 1.0 and math.isclose(plain[-1] / f[-1], 8.0)


def _brute(x, u, t, k, p, m):
    """Over the whole order of the row, by the definition."""
    order = sorted(range(len(x)), key=lambda i: (-x[i], i))
    w = [math.exp((v - max(x)) / t) for v in x]
    order = order[:k] if 0 < k else order
    if p < 1:
        total = sum(w[i] for i in order)
        order = next(order[:n] for n in range(1, len(order) + 1) if sum(w[i] for i in order[:n]) >= p * total or n == len(order))
    order = [i for i in order if w[i] >= m]
    total = sum(w[i] for i in order)
    return next(i for i in sorted(order) if sum(w[j] for j in order if j <= i) > u * total)


def test_sample_against_the_definition():
    g = np.random.default_rng(3)
    for t, k, p, m in itertools.product((0.5, 1.3), (0, 1, 4), (0.3, 0.9, 1.0), (0.0, 0.1)):
        for _ in range(8):
            x, u = np.round(2 * g.standard_normal(12), 1), g.random()
            token, prob, kept, margin = do.sample(x, u, t, k, p, m)
            if margin > 1e-9:
                assert token == _brute(list(x), u, t, k, p, m) and token in kept and 0 < prob <= 1


def test_sample_draws_with_its_probabilities():
    x = np.log(np.array([1.0, 5.0, 2.0, 2.0]))
    got = [do.sample(x, (i + 0.5) / 1000)[0] for i in range(1000)]
    assert [got.count(i) for i in range(4)] == [100, 500, 200, 200]
    assert do.sample(x, 0.5, top_k=2)[2] == [1, 2] and do.sample(x, 0.5, top_p=0.71)[2] == [1, 2, 3]
    assert do.sample(np.full(5, -np.inf), 0.5)[0] == -1 and do.sample(x, 0.0, temperature=0.0)[0] == 1
