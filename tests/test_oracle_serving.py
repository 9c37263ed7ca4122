"""The serving oracle against brute force and its own definitions (no GPU)."""
import numpy as np
import pytest

from oracle import serving_oracle as so


@pytest.mark.parametrize("page,dim", [(64, 64), (128, 128), (256, 64), (64, 256)])
def test_the_layouts_are_permutations(page, dim):
    for place in (so.k_place, so.v_place):
        assert np.array_equal(np.sort(place(page, dim).ravel()), np.arange(page * dim))


def test_layout_as_the_header_writes_it():
    page, dim = 128, 128
    k, v = so.k_place(page, dim), so.v_place(page, dim)
    n = np.arange(page * dim)
    # K: [tile][u][d / 64][d % 64 / 16][g][i][d % 16]
    tile, u, c, quarter, g, i, e = np.unravel_index(n, (page // 64, 4, dim // 64, 4, 4, 4, 16))
    assert np.array_equal(k[64 * tile + 16 * g + 4 * u + i, 64 * c + 16 * quarter + e], n)
    # V: [tile][d / 16][g][d % 16][t % 16]
    tile, dt, g, m, e = np.unravel_index(n, (page // 64, dim // 16, 4, 16, 16))
    assert np.array_equal(v[64 * tile + 16 * g + e, 16 * dt + m], n)


def test_written_at_once_is_within_half_a_step():
    g = np.random.default_rng(1)
    c = so.Cache(4, 2, 64, 64)
    x = g.standard_normal((150, 2, 64)).astype(np.float32)
    c.write([3, 0, 2], 0, x)
    step = np.repeat(c.scale[[3, 0, 2]], 64, axis=0)[:150]
    assert (np.abs(c.dense([3, 0, 2], 150) - x) <= 0.5001 * step[..., None]).all()


@pytest.mark.parametrize("growth", [1.001, 1.05, 1.9, 7.0])
def test_written_token_by_token_is_within_a_step(growth):
    """The promise of the header: doubling keeps what repeated rounding does below one step."""
    g = np.random.default_rng(2)
    c = so.Cache(1, 1, 64, 64)
    x = (g.standard_normal((64, 1, 64)) * growth ** np.arange(64)[:, None, None] * 1e-20).astype(np.float32)
    for t in range(64):
        c.write([0], t, x[t:t + 1])
    assert (np.abs(c.dense([0], 64) - x) <= c.scale[0, 0]).all()
    assert c.scale[0, 0] <= 2.0 * np.abs(x).max() / 127 * 1.0001


def test_zeros_and_non_finite_values():
    c = so.Cache(1, 1, 64, 64)
    c.write([0], 0, np.zeros((3, 1, 64), np.float32))
    assert c.scale[0, 0] > 0 and (c.dense([0], 3) == 0).all()
    bad = np.ones((1, 1, 64), np.float32)
    bad[0, 0, 5] = np.inf
    c.write([0], 3, bad)
    assert np.isnan(c.scale[0, 0])
    c.write([0], 0, np.ones((1, 1, 64), np.float32))
    assert np.isfinite(c.scale[0, 0])


@pytest.mark.parametrize("causal,window", [(True, 0), (True, 3), (False, 0), (False, 2)])
def test_attention_against_softmax_of_the_full_map(causal, window):
    g = np.random.default_rng(3)
    n, kv, n_q, n_kv, dim = 5, 9, 4, 2, 8
    q, k, v = g.standard_normal((n, n_q, dim)), g.standard_normal((kv, n_kv, dim)), g.standard_normal((kv, n_kv, dim))
    out, lse, _, _ = so.attention(q, k, v, 0.3, causal, window)
    for h in range(n_q):
        z = 0.3 * q[:, h] @ k[:, h // 2].T
        for i in range(n):
            for t in range(kv):
                p = kv - n + i
                if (causal and t > p) or (window and t <= p - window):
                    z[i, t] = -np.inf
        e = np.exp(z)
        assert np.allclose(out[:, h], e @ v[:, h // 2] / e.sum(1, keepdims=True))
        assert np.allclose(lse[:, h], np.log(e.sum(1)))


def test_attention_of_rows_that_see_nothing():
    out, lse, _, _ = so.attention(np.ones((4, 1, 8)), np.ones((2, 1, 8)), np.ones((2, 1, 8)), 1.0)
    assert (out[:2] == 0).all() and (lse[:2] == -np.inf).all() and (out[2:] == 1).all()


def test_linear_against_a_loop():
    g = np.random.default_rng(4)
    planes = g.integers(0, 1 << 32, (2, 3, 2), dtype=np.uint32)
    coefs = g.standard_normal((3, 3, 2)).astype(np.float16)
    x = g.standard_normal((2, 64))
    want = np.zeros((2, 3))
    for t in range(2):
        for r in range(3):
            for c in range(64):
                w = float(coefs[0, r, c // 32])
                for i in range(2):
                    w += float(coefs[i + 1, r, c // 32]) * (int(planes[i, r, c // 32]) >> (c % 32) & 1)
                want[t, r] += w * x[t, c]
    assert np.allclose(so.linear(planes, coefs, 32, x)[0], want)
