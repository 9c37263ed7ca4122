"""Attention on the GPU over pages of V whose scales are far apart, and beside pages that a query does not see.

Tolerance, in the notation of test_gpu_serving: p_t the softmax, s_t the scale of V of token t's page, S = sum p |v| of the row, N its tokens.
Scores carry z as there, probabilities are rounded to fp16 (2^-11 of each, S in all), sums of N terms in fp32 cost (N + 16) e S, the result u.
A probability below fp16's normal range has an absolute error instead.  For few rows it is 2^-25 of the largest probability's place, which
the page's scale and a code (at most 128) multiply: 2^-18 max p sum s.  For many rows p s together is rounded, in units of which the row's largest p s is at least
2^7: 2^-25 2^-7 128 max(p s) = 2^-25 max(p s) for each of N tokens.
"""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from test_gpu_serving import E, U, Sequences, _attend, _np, _tokens, dev  # noqa: F401

pytestmark = pytest.mark.gpu

# the largest magnitudes of the pages of V, in order; 0 is a page of zeros
PAGES = {"zeros behind 1e9": [1e9, 0, 1.0], "zeros behind 1e11": [3e11, 0, 1.0, 0], "zeros behind 1e20": [1.0, 1e20, 0, 0.01],
         "falling": [1e3, 1e-16, 1e-30, 0], "rising": [0, 1e-30, 1e-16, 1.0, 1e16, 1e30], "saw": [1.0, 1e-6, 1e6, 1e-6, 1.0, 1e-12, 1.0],
         "far": [1e30, 1.0, 1e-30, 1.0, 1e30, 1e-30], "alike": [1.0, 1.5, 0.7, 2.0]}


def _fill(seq, mags, kv, kind, loud=1.0):
    """kv tokens whose pages of V have the magnitudes in turn."""
    n_kv, dim, page = seq.n_kv, seq.dim, seq.page
    K, V = loud * _tokens(kv, n_kv, dim, kind, 1, seq.dev), _tokens(kv, n_kv, dim, "f32", 2, seq.dev)
    mag = torch.tensor([mags[t // page % len(mags)] for t in range(kv)], device=seq.dev)[:, None, None]
    V = (V / 8 * mag).to(K.dtype)
    seq.write([kv], K, V)


def _check_row_by_row(seq, Q, kind, scale, causal, window, out, hidden=()):
    """out against 64 bits, each row by what it sees."""
    kv, n, dim, group = seq.len[0], len(Q), seq.dim, Q.shape[1] // seq.n_kv
    many = n * group > 32
    k, v = seq.k.dense(seq.table[0], kv), seq.v.dense(seq.table[0], kv)
    s = np.stack([seq.v.scale[seq.table[0, t // seq.page]] for t in range(kv)]).astype(np.float64)        # token, head
    q, got = _np(Q), _np(out)
    at, t = np.arange(kv - n, kv)[:, None], np.arange(kv)[None, :]
    seen = np.ones((n, kv), bool)
    if causal:
        seen &= t <= at
    if window:
        seen &= t > at - window
    for page in hidden:
        seen[:, page * seq.page:(page + 1) * seq.page] = False
    assert seen.any(1).all()
    worst = 0.0
    for h in range(Q.shape[1]):
        g = h // group
        z = np.where(seen, scale * (q[:, h] @ k[:, g].T), -np.inf)
        reach = np.where(seen, abs(scale) * (np.abs(q[:, h]) @ np.abs(k[:, g]).T), 0).max(1)
        p = np.exp(z - z.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        want, size = p @ v[:, g], p @ np.abs(v[:, g])
        zerr = (2 * (dim + 16) * E * reach + 2.0 ** -22)[:, None]
        if many:
            small = kv * 2.0 ** -25 * (p * s[:, g]).max(1)
        else:
            small = 2.0 ** -18 * p.max(1) * (seen * s[:, g]).sum(1)
        tol = (2.0 ** -11 + 2 * zerr) * 1.01 * size + U[kind] * np.abs(want) + (kv + 16) * E * size + small[:, None] + 1e-37
        off = np.abs(got[:, h] - want) / tol
        assert (off <= 1).all(), (h, np.argwhere(~(off <= 1))[:4], np.nanmax(off), np.isnan(got[:, h]).sum())
        worst = max(worst, off.max())
    return worst


@pytest.mark.parametrize("name", list(PAGES))
@pytest.mark.parametrize("n_q,n_kv,dim,page,rows,causal,window,times", [
    (2, 1, 128, 64, 0, True, 0, 1),               # a prompt: early rows see the first pages alone
    (1, 1, 64, 64, 70, False, 0, 1),              # all rows see all pages
    (4, 2, 128, 64, 0, True, 40, 1),              # a window: most rows see one or two pages, other rows of a wavefront others
    (1, 1, 256, 64, 130, True, 100, 2),
    (3, 1, 64, 128, 40, True, 0, 9),              # long enough to be split
    (2, 2, 128, 64, 3, True, 0, 2),               # few rows
    (1, 1, 128, 64, 1, True, 0, 9),
])
def test_attention_over_scales_far_apart(dev, name, n_q, n_kv, dim, page, rows, causal, window, times):  # noqa: F811
    print(f"scales {name}: heads={n_q}/{n_kv} dim={dim} page={page} rows={rows} window={window} times={times}", flush=True)
    mags = PAGES[name]
    kv = page * len(mags) * times - 5
    seq = Sequences(dev, 1, n_kv, dim, page, kv, 23)
    _fill(seq, mags, kv, "bf16")
    n = rows or kv
    Q = torch.randn((n, n_q, dim), generator=torch.Generator().manual_seed(5)).bfloat16().to(dev)
    scale = 1.0 / dim ** 0.5
    out, _ = _attend(seq, Q, [n], scale, causal, window)
    _check_row_by_row(seq, Q, "bf16", scale, causal, window, out)


@pytest.mark.parametrize("name", ["far", "falling", "rising"])
def test_a_large_page_of_little_weight(dev, name):  # noqa: F811
    """Scores so far apart that pages of large values have no weight: what counts are the rows' own largest products."""
    dim = 128
    kv = 64 * len(PAGES[name])
    seq = Sequences(dev, 1, 1, dim, 64, kv, 29)
    _fill(seq, PAGES[name], kv, "bf16", loud=6.0)
    Q = (6 * torch.randn((kv, 1, dim), generator=torch.Generator().manual_seed(5))).bfloat16().to(dev)
    scale = 1.0 / dim ** 0.5
    out, _ = _attend(seq, Q, [kv], scale)
    _check_row_by_row(seq, Q, "bf16", scale, True, 0, out)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("huge", [1e20, 1e-25, 0.0])
def test_attention_does_not_look_at_the_scale_of_page_0(dev, dim, huge):  # noqa: F811
    """Table entries outside the cache, whatever the scales of the cache's first page: its tokens are nobody's here."""
    kv, n = 64 * 6, 64 * 6
    seq = Sequences(dev, 1, 1, dim, 64, kv, 31, spare=3)
    free = next(iter(set(range(6 + 3)) - set(seq.table[0].tolist())))
    seq.table[0][seq.table[0] == 0] = free         # page 0 is nobody's
    _fill(seq, [1.0, 1.0], kv, "bf16")
    Q = torch.randn((n, 1, dim), generator=torch.Generator().manual_seed(5)).bfloat16().to(dev)
    scale, hidden = 1.0 / dim ** 0.5, (1, 4)
    table = seq.table_d
    for page in hidden:
        table[0, page] = -1
    outs = []
    for value in (0.01, huge):
        seq.cache.k_scale[0], seq.cache.v_scale[0] = value, value
        outs.append(_attend(seq, Q, [n], scale, table=table)[0])
    assert torch.equal(outs[0], outs[1])
    _check_row_by_row(seq, Q, "bf16", scale, True, 0, outs[1], hidden)


@pytest.mark.parametrize("dim", [64, 128])
def test_hidden_pages_of_large_values_change_nothing(dev, dim):  # noqa: F811
    """Under a window, large values in pages that a row does not see leave its bits alone, also where other rows of its wavefront see them."""
    kv, n, window = 64 * 6, 200, 64
    Q = torch.randn((n, 1, dim), generator=torch.Generator().manual_seed(5)).bfloat16().to(dev)
    outs = []
    for large in (1.0, 1e20):
        seq = Sequences(dev, 1, 1, dim, 64, kv, 37)
        _fill(seq, [1.0, 1.0, 1.0, large, 1.0, 1.0], kv, "bf16")
        outs.append(_attend(seq, Q, [n], 1.0 / dim ** 0.5, window=window)[0])
        _check_row_by_row(seq, Q, "bf16", 1.0 / dim ** 0.5, True, window, outs[-1])
    at = torch.arange(kv - n, kv, device=dev)
    blind = (at < 64 * 3) | (at - window >= 64 * 4 - 1)
    assert blind.any() and torch.equal(outs[0][blind], outs[1][blind])
