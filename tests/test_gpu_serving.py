"""Serving on the GPU, through the binding, against the numpy oracle: the product with bias, activation and residual, the 8-bit
cache as it is written and read, and attention over it.

Tolerances.  u = 2^-11 (float16) or 2^-8 (bfloat16) is the largest relative error of one rounding to the type, e = 2^-24 that of
fp32.  Product: What is rounded once to fp16 (w = 2^-11 of it), a sum of d products in any order costs at most d e, the result is
rounded once: |error| <= (w + (d + 16) e) S + u |y|, S = sum |What| |x| + |bias|, times the activation's steepest slope (below 1.13), and
over all values (roundings are independent) at most u + w of the norm of what was rounded.
Attention: scores carry (dim + 16) e times max |scale| sum |q| |k| (plus |log2| terms of the exponential, the same size), probabilities
an error of u16 = 2^-11 each from their rounding to fp16 (or 2^-25 of the largest), the result u.
"""
import ctypes

import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2602_04163_amd import binding as bq

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
E, W16 = 2.0 ** -24, 2.0 ** -11


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    bq.load()
    return torch.device("cuda:0")


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


# ------------------------------------------------------------------ the product

def _layer(d_out, d_in, bits, group, seed):
    g = np.random.default_rng(seed)
    planes = g.integers(0, 1 << 32, (bits, d_out, d_in // 32), dtype=np.uint32)
    coefs = (g.standard_normal((bits + 1, d_out, d_in // group)) * 0.05).astype(np.float16)
    return planes, coefs


def _on(planes, coefs, dev):
    return torch.from_numpy(planes.view(np.int32)).to(dev), torch.from_numpy(coefs).to(dev)


def _check_linear(y, want, size, kind, d_in, residual=None):
    u = U[kind]
    got = _np(y)
    tol = 1.13 * (W16 + (d_in + 16) * E) * size + u * np.abs(want) + 2.0 ** -24 * (1 + d_in)
    if residual is not None:
        tol += E * np.abs(residual)
    assert (np.abs(got - want) <= tol).all(), np.max(np.abs(got - want) / tol)
    base = want if residual is None else np.concatenate([want, want - residual])
    assert np.linalg.norm(got - want) <= (u + W16) * np.linalg.norm(base) + 2.0 ** -20 * np.sqrt(want.size)


@pytest.mark.parametrize("bits,group,d_out,d_in,n,kind,act,bias,residual", [
    (2, 128, 48, 512, 1, "bf16", "none", True, False),
    (2, 64, 33, 640, 1, "f16", "silu", False, True),
    (1, 32, 16, 32, 2, "f16", "none", True, True),
    (3, 32, 7, 96, 3, "bf16", "relu", False, False),
    (4, 64, 130, 1088, 5, "f16", "gelu", True, False),
    (2, 96, 65, 288, 15, "bf16", "gelu_tanh", True, True),
    (3, 128, 64, 4096, 16, "f16", "none", False, True),
    (1, 256, 257, 768, 17, "bf16", "silu", True, False),
    (2, 32, 31, 8224, 31, "f16", "relu", False, False),
    (4, 32, 100, 2080, 32, "bf16", "none", True, True),
    (2, 128, 300, 1152, 33, "f16", "gelu", False, True),
    (3, 64, 64, 64, 64, "bf16", "none", False, False),
    (2, 64, 200, 1984, 65, "bf16", "silu", True, True),
    (3, 256, 513, 1280, 127, "f16", "gelu_tanh", True, False),
    (2, 128, 256, 512, 128, "bf16", "none", True, True),
    (1, 32, 255, 416, 129, "f16", "none", False, False),
    (4, 128, 384, 640, 200, "bf16", "relu", True, False),
    (2, 128, 513, 2176, 257, "f16", "none", False, True),
    (2, 64, 1024, 1088, 515, "bf16", "silu", True, True),
    (3, 128, 770, 896, 1025, "f16", "gelu", False, False),
    (2, 256, 1537, 768, 2049, "bf16", "none", True, False),
    (1, 64, 2050, 320, 1100, "f16", "none", True, False),
    (4, 64, 1030, 448, 1500, "bf16", "none", False, True),
])
def test_linear(dev, bits, group, d_out, d_in, n, kind, act, bias, residual):
    print(f"linear k={bits} g={group} {d_out}x{d_in} n={n} {kind} {act}", flush=True)
    planes, coefs = _layer(d_out, d_in, bits, group, d_out + d_in + n)
    g = torch.Generator().manual_seed(n)
    t = TYPES[kind]
    x = (torch.randn((n, d_in), generator=g) * torch.exp(0.5 * torch.randn(d_in, generator=g))).to(t)
    b = torch.randn(d_out, generator=g).to(t) if bias else None
    r = (4 * torch.randn((n, d_out), generator=g)).to(t) if residual else None
    want, size = so.linear(planes, coefs, group, _np(x), None if b is None else _np(b), act, None if r is None else _np(r))
    p, c = _on(planes, coefs, dev)
    on = lambda v: None if v is None else v.to(dev)  # noqa: E731
    y = bq.bpdq_linear(p, c, group, on(x), bias=on(b), act=act, residual=on(r))
    _check_linear(y, want, size, kind, d_in, None if r is None else _np(r))
    assert torch.equal(y, bq.bpdq_linear(p, c, group, on(x), bias=on(b), act=act, residual=on(r)))


# tokens, columns and rows for which each of the kernels is chosen: few tokens (2, 3, 5 and 8 row tiles; twice 16 tokens with 2, 3 and 5), tiles of
# 128 x 64, 128 x 128, 256 x 128 and 256 x 256
@pytest.mark.parametrize("n,d_in,d_out", [(513, 256, 130), (257, 256, 520), (65, 256, 3100), (65, 256, 4100), (1500, 256, 130),
                                          (700, 256, 520), (513, 256, 1000), (257, 1024, 5000), (300, 512, 8200), (1025, 256, 5000),
                                          (1025, 256, 8200)])
@pytest.mark.parametrize("bits,group,kind", [(1, 128, "bf16"), (2, 64, "f16"), (3, 32, "bf16"), (4, 128, "f16"), (2, 0, "bf16")])
def test_linear_kernels(dev, n, d_in, d_out, bits, group, kind):
    """Every kernel with groups of four words, of two and of one; with one word more to a row (group 0), so that rows are not 16 bytes and
    the last columns end inside a tile."""
    if group == 0:
        d_in, group = d_in + 32, (96 if (d_in + 32) % 96 == 0 else 32)
    print(f"linear kernels k={bits} g={group} {d_out}x{d_in} n={n} {kind}", flush=True)
    planes, coefs = _layer(d_out, d_in, bits, group, n)
    g = torch.Generator().manual_seed(n)
    x = (torch.randn((n, d_in), generator=g) * torch.exp(0.5 * torch.randn(d_in, generator=g))).to(TYPES[kind])
    b = torch.randn(d_out, generator=g).to(TYPES[kind])
    r = (4 * torch.randn((n, d_out), generator=g)).to(TYPES[kind])
    want, size = so.linear(planes, coefs, group, _np(x), _np(b), "relu", _np(r))
    p, c = _on(planes, coefs, dev)
    y = bq.bpdq_linear(p, c, group, x.to(dev), bias=b.to(dev), act="relu", residual=r.to(dev))
    _check_linear(y, want, size, kind, d_in, _np(r))
    assert torch.equal(y, bq.bpdq_linear(p, c, group, x.to(dev), bias=b.to(dev), act="relu", residual=r.to(dev)))


@pytest.mark.parametrize("n,d_in,pad,shift", [(1, 512, 3, 1), (20, 288, 8, 0), (20, 1024, 8, 8), (70, 512, 5, 3), (300, 2048, 8, 4),
                                              (600, 640, 1, 1), (1030, 1024, 16, 8)])
def test_linear_strides_and_alignment(dev, n, d_in, pad, shift):
    """Rows of X, of the residual and of Y with gaps, off 16 bytes; nothing but Y's rows is written; Y over the residual."""
    print(f"linear strides n={n} d_in={d_in} pad={pad} shift={shift}", flush=True)
    d_out, bits, group, t = 67, 2, 32, torch.bfloat16
    planes, coefs = _layer(d_out, d_in, bits, group, n)
    g = torch.Generator().manual_seed(n)
    flat = torch.full(((n + 1) * (d_in + pad) + shift,), float("nan"), dtype=t)
    X = flat[shift:shift + n * (d_in + pad)].view(n, d_in + pad)[:, :d_in]
    X.copy_(torch.randn((n, d_in), generator=g))
    store = torch.full((n, d_out + pad), 7.0, dtype=t)
    store[:, :d_out] = torch.randn((n, d_out), generator=g).to(t)
    want, size = so.linear(planes, coefs, group, _np(X), None, "silu", _np(store[:, :d_out]))
    p, c = _on(planes, coefs, dev)
    fd, sd = flat.to(dev), store.to(dev)
    Xd = fd[shift:shift + n * (d_in + pad)].view(n, d_in + pad)[:, :d_in]
    Y = sd[:, :d_out]
    bq.bpdq_linear(p, c, group, Xd, act="silu", residual=Y, Y=Y)
    _check_linear(Y, want, size, "bf16", d_in, _np(store[:, :d_out]))
    assert (sd[:, d_out:] == 7.0).all()
    # planes off 16 bytes: the same values
    shifted = torch.empty(p.numel() + 1, dtype=torch.int32, device=dev)
    shifted[1:] = p.flatten()
    again = bq.bpdq_linear(shifted[1:].view(p.shape), c, group, Xd, act="silu")
    assert torch.equal(again, bq.bpdq_linear(p, c, group, Xd, act="silu"))


@pytest.mark.parametrize("n", [1, 16, 40, 300, 1100])
def test_linear_keeps_what_is_not_finite_in_its_row(dev, n):
    """A NaN or infinity in a token reaches that token's results alone; what lies behind X's last column is not read."""
    planes, coefs = _layer(80, 544, 3, 32, 5)
    p, c = _on(planes, coefs, dev)
    x = torch.randn((n, 544), generator=torch.Generator().manual_seed(1)).half().to(dev)
    clean = bq.bpdq_linear(p, c, 32, x)
    x[n // 2, 543] = float("inf")
    y = bq.bpdq_linear(p, c, 32, x)
    assert not torch.isfinite(y[n // 2]).any()
    keep = torch.arange(n, device=dev) != n // 2
    assert torch.equal(y[keep], clean[keep])


@pytest.mark.parametrize("n", [1, 3, 20, 70, 260])
def test_linear_of_tokens_of_all_sizes(dev, n):
    """bfloat16 reaches far beyond float16: tokens from 2^-120 to 2^100, each as exact as it would be alone; zeros and denormals."""
    d_in, d_out = 288, 48
    planes, coefs = _layer(d_out, d_in, 2, 96, n)
    g = torch.Generator().manual_seed(n)
    x = torch.randn((n, d_in), generator=g) * torch.exp(torch.randn(d_in, generator=g))
    power = torch.linspace(-120, 100, n).round() if n > 1 else torch.tensor([-120.0])
    x = (x * torch.exp2(power)[:, None]).bfloat16()
    if n > 3:
        x[1] = 0
        x[2] = 1e-39 * torch.randn(d_in, generator=g)
    want, size = so.linear(planes, coefs, 96, _np(x))
    y = _np(bq.bpdq_linear(*_on(planes, coefs, dev), 96, x.to(dev)))
    tol = (W16 + (d_in + 16) * E) * size + U["bf16"] * np.abs(want) + 2.0 ** -29 * np.abs(_np(x)).max(1, keepdims=True) * d_in * 0.3 + 1e-40
    assert (np.abs(y - want) <= tol).all(), np.max(np.abs(y - want) / tol)


def test_linear_is_the_dequantized_product(dev):
    """Tokens that are unit vectors give the columns of What, rounded to fp16 and then to the type."""
    planes, coefs = _layer(64, 256, 4, 64, 9)
    p, c = _on(planes, coefs, dev)
    w = bq.bpdq_dequant_fp16(p, c, 64)
    for t in (torch.float16, torch.bfloat16):
        y = bq.bpdq_linear(p, c, 64, torch.eye(256, device=dev, dtype=t))
        assert torch.equal(y, w.t().half().to(t))


def test_linear_refuses_tensors(dev):
    planes, coefs = _layer(32, 64, 2, 32, 1)
    p, c = _on(planes, coefs, dev)
    x = torch.zeros((2, 64), dtype=torch.float16, device=dev)
    for bad in (lambda: bq.bpdq_linear(p, c, 32, x.float()), lambda: bq.bpdq_linear(p, c, 32, x[:, :32]),
                lambda: bq.bpdq_linear(p, c, 32, x, act="tanh"), lambda: bq.bpdq_linear(p, c, 64, x),
                lambda: bq.bpdq_linear(p, c, 32, x, bias=torch.zeros(31, dtype=torch.float16, device=dev)),
                lambda: bq.bpdq_linear(p, c, 32, x, bias=torch.zeros(32, device=dev)),
                lambda: bq.bpdq_linear(p, c, 32, x, residual=torch.zeros((3, 32), dtype=torch.float16, device=dev)),
                lambda: bq.bpdq_linear(p, c, 32, x.cpu()), lambda: bq.bpdq_linear(p, c, 32, x.t())):
        with pytest.raises(bq.BpdqError):
            bad()
    assert bq.bpdq_linear(p, c, 32, x[:0]).shape == (0, 32)


# ------------------------------------------------------------------ the cache

class Sequences:
    """A cache on the GPU and its oracle, with pages dealt in no order."""

    def __init__(self, dev, n_seq, n_kv, dim, page, most, seed, spare=2):
        self.dev, self.page, self.dim, self.n_kv = dev, page, dim, n_kv
        width = -(-most // page)
        n_pages = n_seq * width + spare
        g = np.random.default_rng(seed)
        self.table = g.permutation(n_pages)[:n_seq * width].reshape(n_seq, width).astype(np.int32)
        self.k, self.v = (so.Cache(n_pages, n_kv, page, dim) for _ in range(2))
        self.cache = bq.KvCache.empty(n_pages, n_kv, dim, page, dev)
        for t in (self.cache.k, self.cache.v):
            t.random_(0, 256)                        # what a page held before
        for t in (self.cache.k_scale, self.cache.v_scale):
            t.fill_(float("nan"))
        self.len = [0] * n_seq

    def ints(self, v):
        return torch.tensor(list(v), dtype=torch.int32, device=self.dev)

    @property
    def table_d(self):
        return torch.from_numpy(self.table).to(self.dev)

    def write(self, counts, K, V, max_tok=None, pos=None):
        pos = list(self.len) if pos is None else pos
        start = np.concatenate([[0], np.cumsum(counts)])
        bq.bpdq_kv_write(self.cache, self.table_d, self.ints(pos), self.ints(start), K, V, max(counts) if max_tok is None else max_tok)
        Kn, Vn = K.float().cpu().numpy(), V.float().cpu().numpy()
        for b, n in enumerate(counts):
            self.k.write(self.table[b], pos[b], Kn[start[b]:start[b] + n])
            self.v.write(self.table[b], pos[b], Vn[start[b]:start[b] + n])
            self.len[b] = pos[b] + n

    def check(self):
        """Codes and scales are the oracle's, bit for bit, in every slot that has been written."""
        for mine, code, scale, place in ((self.k, self.cache.k, self.cache.k_scale, so.k_place(self.page, self.dim)),
                                         (self.v, self.cache.v, self.cache.v_scale, so.v_place(self.page, self.dim))):
            code, scale = code.cpu().numpy().reshape(len(code), self.n_kv, -1), scale.cpu().numpy()
            for b, n in enumerate(self.len):
                for j in range(-(-n // self.page)):
                    p, slots = self.table[b, j], min(self.page, n - j * self.page)
                    assert np.array_equal(scale[p], mine.scale[p], equal_nan=True)
                    got = code[p][:, place][:, :slots]
                    ok = np.isfinite(mine.scale[p])
                    assert np.array_equal(got[ok], mine.code[p][:, :slots][ok])


def _tokens(n, n_kv, dim, kind, seed, dev, grow=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, n_kv, dim), generator=g) * torch.exp(0.5 * torch.randn((n_kv, dim), generator=g))
    x *= torch.exp(grow * torch.randn((n, 1, 1), generator=g))
    return x.to(TYPES[kind]).to(dev)


@pytest.mark.parametrize("n_kv,dim,page,kind,steps", [
    (1, 64, 64, "f32", [[1], [1], [1], [61], [1], [130]]),
    (3, 128, 64, "bf16", [[70, 0, 5], [1, 1, 1], [0, 3, 200], [1, 64, 1], [17, 1, 0]]),
    (2, 256, 64, "f16", [[15, 64], [2, 1], [65, 127], [1, 1]]),
    (4, 64, 128, "bf16", [[127, 128, 129], [1, 1, 1], [1, 1, 1], [300, 2, 1]]),
    (1, 128, 256, "f16", [[255, 3], [1, 1], [1, 1], [257, 250], [3, 9]]),
    (5, 256, 256, "f32", [[3, 256], [16, 1], [240, 255]]),
])
def test_cache_as_it_is_written(dev, n_kv, dim, page, kind, steps):
    print(f"cache write heads={n_kv} dim={dim} page={page} {kind}", flush=True)
    most = max(sum(s[b] for s in steps) for b in range(len(steps[0])))
    seq = Sequences(dev, len(steps[0]), n_kv, dim, page, most, dim + page)
    for i, counts in enumerate(steps):
        n = sum(counts)
        seq.write(counts, _tokens(n, n_kv, dim, kind, 10 * i, dev, 1.0), _tokens(n, n_kv, dim, kind, 10 * i + 1, dev, 1.0))
        seq.check()
    # read back from anywhere, in every type
    for kind2, u in U.items():
        pos = [n // 3 for n in seq.len]
        back = [n - p for n, p in zip(seq.len, pos)]
        start = np.concatenate([[0], np.cumsum(back)])
        K, V = bq.bpdq_kv_read(seq.cache, seq.table_d, seq.ints(pos), seq.ints(start), int(start[-1]), max(back), TYPES[kind2])
        for got, mine in ((K, seq.k), (V, seq.v)):
            want = np.concatenate([mine.dense(seq.table[b], seq.len[b])[pos[b]:] for b in range(len(pos))])
            # the product's own rounding to fp32 comes before that to the type
            assert (np.abs(_np(got) - want) <= (u + E) * np.abs(want) + 2.0 ** -25 * (kind2 == "f16")).all()


@pytest.mark.parametrize("kind,pad,shift", [("bf16", 3, 1), ("f16", 8, 8), ("f32", 1, 1), ("bf16", 16, 4)])
def test_cache_of_strided_rows(dev, kind, pad, shift):
    """Keys and values as slices of one product's rows, off 16 bytes too; the read fills slices and nothing beside them."""
    n, n_kv, dim, page = 75, 2, 64, 64
    row = 2 * n_kv * dim + pad
    flat = torch.randn(n * row + shift, generator=torch.Generator().manual_seed(3)).to(TYPES[kind]).to(dev)
    rows = flat[shift:].view(n, row)
    K, V = rows[:, :n_kv * dim].unflatten(1, (n_kv, dim)), rows[:, n_kv * dim:2 * n_kv * dim].unflatten(1, (n_kv, dim))
    seq = Sequences(dev, 1, n_kv, dim, page, n, 1)
    seq.write([n], K, V)
    seq.check()
    out = torch.full_like(flat, 7.0)
    into = out[shift:].view(n, row)
    K2, V2 = into[:, :n_kv * dim].unflatten(1, (n_kv, dim)), into[:, n_kv * dim:2 * n_kv * dim].unflatten(1, (n_kv, dim))
    bq.bpdq_kv_read(seq.cache, seq.table_d, seq.ints([0]), seq.ints([0, n]), n, dtype=TYPES[kind], K=K2, V=V2)
    want = bq.bpdq_kv_read(seq.cache, seq.table_d, seq.ints([0]), seq.ints([0, n]), n, dtype=TYPES[kind])
    assert torch.equal(K2, want[0]) and torch.equal(V2, want[1])
    assert (into[:, 2 * n_kv * dim:] == 7.0).all() and (out[:shift] == 7.0).all()


def test_cache_extremes(dev):
    """Zeros, denormals, the type's largest values, a NaN and an infinity, and a page that is written anew."""
    n_kv, dim = 2, 64
    seq = Sequences(dev, 1, n_kv, dim, 64, 192, 4)
    x = torch.zeros((4, n_kv, dim), device=dev)
    seq.write([4], x, x)
    seq.check()
    x = torch.full((3, n_kv, dim), 1e-42, device=dev)
    x[1, 0, 3] = 1e-20
    seq.write([3], x, x)
    seq.check()
    x = torch.full((2, n_kv, dim), 3.0e38, device=dev)
    x[:, 1] = 1e-10
    seq.write([2], x, -x)
    seq.check()
    bad = torch.ones((1, n_kv, dim), device=dev)
    bad[0, 1, 60] = float("nan")
    inf = torch.ones((1, n_kv, dim), device=dev)
    inf[0, 0, 0] = -float("inf")
    seq.write([1], bad, inf)
    seq.check()
    assert torch.isnan(seq.cache.k_scale[seq.table[0, 0], 1]) and torch.isfinite(seq.cache.k_scale[seq.table[0, 0], 0])
    assert torch.isnan(seq.cache.v_scale[seq.table[0, 0], 0])
    seq.write([1], torch.ones_like(bad), torch.ones_like(bad))       # stays poisoned
    seq.check()
    K, _ = bq.bpdq_kv_read(seq.cache, seq.table_d, seq.ints([0]), seq.ints([0, 11]), 11)
    assert torch.isnan(K[:, 1]).all() and torch.isfinite(K[:, 0]).all()
    seq.write([3], torch.randn((3, n_kv, dim), device=dev), torch.randn((3, n_kv, dim), device=dev), pos=[0])
    seq.check()


def test_cache_leaves_out_what_it_must(dev):
    """Pages outside the cache, negative positions, tokens behind the table, rows behind K, more tokens than max_tok: nothing else is
    touched, and reads of such tokens give zeros."""
    n_kv, dim, page = 2, 64, 64
    seq = Sequences(dev, 4, n_kv, dim, page, 128, 6)
    table = seq.table.copy()
    table[1, 1], table[2, 0] = -1, 10 ** 6
    td = torch.from_numpy(table).to(dev)
    K, V = _tokens(400, n_kv, dim, "f32", 1, dev), _tokens(400, n_kv, dim, "f32", 2, dev)
    before = [t.clone() for t in (seq.cache.k, seq.cache.v, seq.cache.k_scale, seq.cache.v_scale)]
    # counts 100 each: sequence 0 runs over its table, 1 into page -1, 2 begins in a page outside, 3 is negative
    pos, start = seq.ints([60, 0, 0, -1]), seq.ints([0, 100, 200, 300, 400])
    bq.bpdq_kv_write(seq.cache, td, pos, start, K, V, 100)
    fresh = {int(table[0, 0]), int(table[0, 1]), int(table[1, 0]), int(table[2, 1])}
    for was, now in zip(before, (seq.cache.k, seq.cache.v, seq.cache.k_scale, seq.cache.v_scale)):
        for p in range(len(now)):
            same = torch.equal(now[p].view(torch.uint8), was[p].view(torch.uint8))
            # the page that sequence 0 goes on in has no scale yet (NaN), and keeps that
            assert same == (p not in fresh or (p == int(table[0, 0]) and now.dim() == 2)), p
    k, v = bq.bpdq_kv_read(seq.cache, td, pos, start, 400, 100)
    assert (k[68:100] == 0).all() and (k[164:200] == 0).all() and (v[200:264] == 0).all()
    step = seq.cache.k_scale[int(table[1, 0])][None, :, None]
    assert ((k[100:164] - K[100:164]).abs() <= 0.5001 * step).all()
    # rows behind K and counts above max_tok are cut: sequence 0 may fill 10 of its tokens, sequence 1 none
    for t, was in zip((seq.cache.k, seq.cache.v, seq.cache.k_scale, seq.cache.v_scale), before):
        t.copy_(was)
    bq.bpdq_kv_write(seq.cache, td, seq.ints([0, 0, 0, 0]), seq.ints([0, 30, 30, 30, 30]), K[:30], V[:30], 10)
    a = bq.bpdq_kv_read(seq.cache, td, seq.ints([0] * 4), seq.ints([0, 10, 10, 10, 10]), 10, 10)[0]
    seq2 = Sequences(dev, 1, n_kv, dim, page, 64, 8)
    seq2.write([10], K[:10], V[:10])
    b = bq.bpdq_kv_read(seq2.cache, seq2.table_d, seq2.ints([0]), seq2.ints([0, 10]), 10)[0]
    assert torch.equal(a, b)


def test_cache_refuses_tensors(dev):
    seq = Sequences(dev, 1, 2, 64, 64, 64, 1)
    x = torch.zeros((3, 2, 64), dtype=torch.float16, device=dev)
    pos, start = seq.ints([0]), seq.ints([0, 3])
    for bad in (lambda: bq.bpdq_kv_write(seq.cache, seq.table_d, pos, start, x, x.float()),
                lambda: bq.bpdq_kv_write(seq.cache, seq.table_d, pos, start, x[:, :1], x[:, :1]),
                lambda: bq.bpdq_kv_write(seq.cache, seq.table_d, pos, start, x.double(), x.double()),
                lambda: bq.bpdq_kv_write(seq.cache, seq.table_d.long(), pos, start, x, x),
                lambda: bq.bpdq_kv_write(seq.cache, seq.table_d, pos, pos, x, x),
                lambda: bq.bpdq_kv_write(seq.cache, seq.table_d, pos.cpu(), start, x, x),
                lambda: bq.bpdq_kv_write(seq.cache, seq.table_d, pos, start, x.transpose(1, 2).contiguous().transpose(1, 2), x),
                lambda: bq.bpdq_kv_read(seq.cache, seq.table_d, pos, start, 3, dtype=torch.int32),
                lambda: bq.KvCache(seq.cache.k, seq.cache.v[:2], seq.cache.k_scale, seq.cache.v_scale),
                lambda: bq.KvCache(seq.cache.k.float(), seq.cache.v, seq.cache.k_scale, seq.cache.v_scale)):
        with pytest.raises(bq.BpdqError):
            bad()


# ------------------------------------------------------------------ attention

def _attend(seq, Q, q_counts, scale=None, causal=True, window=0, kind="f16", table=None, lse=True, **kw):
    start = np.concatenate([[0], np.cumsum(q_counts)])
    out = torch.full_like(Q.contiguous(), 3.0)
    L = torch.full(Q.shape[:2], 3.0, device=seq.dev) if lse else None
    bq.bpdq_kv_attention(seq.cache, seq.table_d if table is None else table, seq.ints(seq.len), seq.ints(start), Q, max(q_counts),
                         max(max(seq.len), 1), scale, causal, window, out=out, lse=L, **kw)
    return out, L


def _check_attention(seq, Q, q_counts, kind, scale, causal, window, out, L):
    dim, start = seq.dim, np.concatenate([[0], np.cumsum(q_counts)])
    for b, n in enumerate(q_counts):
        if not n:
            continue
        k, v = seq.k.dense(seq.table[b], seq.len[b]), seq.v.dense(seq.table[b], seq.len[b])
        want, lse, size, reach = so.attention(_np(Q[start[b]:start[b] + n]), k, v, scale, causal, window)
        z = (2 * (dim + 16) * E * reach + 2.0 ** -22)[..., None]      # scores and the exponential's argument
        big = np.abs(v).max() if len(v) else 0.0
        tol = (2.0 ** -11 + 2 * z) * 1.01 * size + U[kind] * np.abs(want) + 2.0 ** -24 * (len(v) + 16) * big + 2.0 ** -24
        got = _np(out[start[b]:start[b] + n])
        assert (np.abs(got - want) <= tol).all(), (b, np.max(np.abs(got - want) / tol))
        if L is not None:
            gl = _np(L[start[b]:start[b] + n])
            empty = np.isinf(lse)
            assert np.array_equal(np.isinf(gl), empty) and (got[empty] == 0).all()
            assert (np.abs(gl[~empty] - lse[~empty]) <= z[..., 0][~empty] + 2.0 ** -20 + 2.0 ** -22 * np.abs(lse[~empty])).all()


@pytest.mark.parametrize("n_q,n_kv,dim,page,kind,kv,q,causal,window", [
    (4, 4, 64, 64, "f16", [1, 2, 63, 64, 65], [1] * 5, True, 0),
    (28, 4, 128, 64, "bf16", [0, 130, 517], [1, 1, 1], True, 0),
    (8, 1, 256, 64, "f16", [70, 200], [1, 1], True, 0),
    (16, 1, 128, 128, "bf16", [300], [1], True, 0),
    (34, 2, 64, 64, "f16", [129, 40], [1, 1], True, 0),               # 17 rows to a key head
    (7, 7, 128, 256, "bf16", [255, 256, 257], [1, 1, 1], True, 0),
    (6, 2, 128, 64, "f16", [100, 1, 64], [5, 1, 0], True, 0),
    (6, 3, 64, 64, "bf16", [2, 70], [6, 9], True, 0),                 # more queries than tokens: the first see nothing
    (4, 2, 128, 64, "bf16", [150, 90], [150, 33], True, 0),
    (5, 5, 64, 128, "f16", [333], [333], True, 0),
    (4, 1, 256, 64, "bf16", [200, 77], [100, 77], True, 0),
    (4, 2, 64, 64, "f16", [300, 64], [20, 64], True, 1),
    (4, 2, 64, 64, "f16", [300, 64], [20, 64], True, 5),
    (4, 2, 128, 64, "bf16", [400, 129], [200, 129], True, 64),
    (3, 1, 128, 64, "f16", [777], [1], True, 100),
    (4, 2, 128, 64, "bf16", [140, 33], [10, 40], False, 0),
    (4, 2, 64, 64, "f16", [140, 33], [10, 40], False, 16),
    (14, 2, 128, 64, "bf16", [3000], [1], True, 0),                   # long enough to be split
    (4, 1, 64, 128, "f16", [2500, 1, 600], [2, 1, 2], True, 0),
    (8, 2, 256, 256, "bf16", [2100], [3], True, 0),
    (2, 1, 128, 64, "f16", [1500], [70], True, 0),
    (2, 2, 64, 64, "bf16", [5000], [45], True, 0),                    # many rows over more tiles than a wavefront has lanes, split
    (3, 1, 128, 256, "f16", [4600, 90], [40, 90], True, 700),
    (33, 1, 256, 64, "bf16", [700], [1], True, 0),                    # 33 rows of one token
    (2, 1, 64, 128, "f16", [900, 0, 300], [129, 3, 64], False, 0),
])
def test_attention(dev, n_q, n_kv, dim, page, kind, kv, q, causal, window):
    print(f"attention heads={n_q}/{n_kv} dim={dim} page={page} {kind} kv={kv} q={q} causal={causal} window={window}", flush=True)
    seq = Sequences(dev, len(kv), n_kv, dim, page, max(kv), sum(kv) + sum(q))
    seq.write(kv, _tokens(sum(kv), n_kv, dim, kind, 1, dev), _tokens(sum(kv), n_kv, dim, kind, 2, dev))
    rows = torch.randn((sum(q), (n_q + 1) * dim), generator=torch.Generator().manual_seed(7)).to(TYPES[kind]).to(dev)
    Q = rows[:, :n_q * dim].unflatten(1, (n_q, dim))
    scale = 1.7 / dim ** 0.5
    out, L = _attend(seq, Q, q, scale, causal, window)
    _check_attention(seq, Q, q, kind, scale, causal, window, out, L)
    again, L2 = _attend(seq, Q, q, scale, causal, window)
    assert torch.equal(again, out) and torch.equal(L, L2)
    out3, _ = _attend(seq, Q, q, scale, causal, window, lse=False)
    assert torch.equal(out3, out)


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("kv,q", [([200], [1]), ([90], [90]), ([2000], [2]), ([500], [300])])
def test_attention_of_large_scores(dev, kind, kv, q):
    """Scores of thousands: one token takes all, nothing overflows; in bfloat16 also queries beyond the range of float16."""
    seq = Sequences(dev, 1, 2, 128, 64, kv[0], 3)
    seq.write(kv, _tokens(kv[0], 2, 128, kind, 1, dev), _tokens(kv[0], 2, 128, kind, 2, dev))
    Q = torch.randn((q[0], 4, 128), generator=torch.Generator().manual_seed(5)) * (1e5 if kind == "bf16" else 3e3)
    Q = Q.to(TYPES[kind]).to(dev)
    scale = 1e-2 if kind == "bf16" else 0.3
    out, L = _attend(seq, Q, q, scale)
    # scores of thousands with fp32 sums: the difference of two of them is known to 2^-24 of their size
    _check_attention(seq, Q, q, kind, scale, True, 0, out, L)


@pytest.mark.parametrize("kv,q", [([150], [1]), ([1400], [1]), ([150], [100]), ([1400], [200])])
def test_attention_does_not_look_at_what_is_hidden(dev, kv, q):
    """Slots behind the last token, pages that nobody sees (NaN scales, or no page at all), and pages of other heads."""
    seq = Sequences(dev, 1, 2, 128, 64, kv[0] + 256, 11)
    seq.write(kv, _tokens(kv[0], 2, 128, "bf16", 1, dev), _tokens(kv[0], 2, 128, "bf16", 2, dev))
    Q = torch.randn((q[0], 4, 128), generator=torch.Generator().manual_seed(5)).bfloat16().to(dev)
    out, _ = _attend(seq, Q, q)
    table = seq.table_d
    table[0, -(-kv[0] // 64):] = -5
    hidden, _ = _attend(seq, Q, q, table=table)
    assert torch.equal(out, hidden)
    # under a window: everything before it may be poisoned
    low = (kv[0] - q[0] + 1 - 64) // 64
    if low > 0:
        want, _ = _attend(seq, Q, q, window=64)
        for p in seq.table[0, :low]:
            seq.cache.k_scale[int(p)] = float("nan")
            seq.cache.v_scale[int(p)] = float("inf")
        got, _ = _attend(seq, Q, q, window=64)
        assert torch.equal(want, got)


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("n_kv,kv,q", [(2, 190, 190), (1, 1500, 60), (2, 190, 5)])
def test_attention_over_a_poisoned_page(dev, which, n_kv, kv, q):
    """A page whose scale is NaN reaches the queries that see one of its tokens, and no others, in that head alone."""
    seq = Sequences(dev, 1, n_kv, 64, 64, kv, 13)
    seq.write([kv], _tokens(kv, n_kv, 64, "f16", 1, dev), _tokens(kv, n_kv, 64, "f16", 2, dev))
    Q = torch.randn((q, 2 * n_kv, 64), generator=torch.Generator().manual_seed(5)).half().to(dev)
    clean, _ = _attend(seq, Q, [q])
    page = (kv - q // 2) // 64
    getattr(seq.cache, which + "_scale")[int(seq.table[0, page]), 0] = float("nan")
    got, _ = _attend(seq, Q, [q])
    sees = torch.arange(kv - q, kv, device=dev) >= 64 * page
    assert torch.isnan(got[sees][:, :2]).all()
    assert torch.equal(got[~sees], clean[~sees]) and torch.equal(got[:, 2:], clean[:, 2:])


@pytest.mark.parametrize("q", [1, 40])
def test_attention_skips_pages_outside_the_cache(dev, q):
    """A table entry outside the cache hides its tokens."""
    kv, dim = 256, 64
    seq = Sequences(dev, 1, 1, dim, 64, kv, 17)
    seq.write([kv], _tokens(kv, 1, dim, "f16", 1, dev), _tokens(kv, 1, dim, "f16", 2, dev))
    Q = torch.randn((q, 1, dim), generator=torch.Generator().manual_seed(5)).half().to(dev)
    table = seq.table_d
    table[0, 1] = 10 ** 8
    got, L = _attend(seq, Q, [q], table=table)
    k, v = seq.k.dense(seq.table[0], kv), seq.v.dense(seq.table[0], kv)
    z = _np(Q[:, 0]) @ k[:, 0].T / dim ** 0.5
    z[:, 64:128] = -np.inf
    z[np.arange(kv)[None, :] > np.arange(kv - q, kv)[:, None]] = -np.inf
    p = np.exp(z - z.max(1, keepdims=True))
    want = p @ v[:, 0] / p.sum(1, keepdims=True)
    assert np.abs(_np(got[:, 0]) - want).max() <= 2.0 ** -9 * np.abs(v).max()


def test_attention_far_into_a_large_cache(dev):
    """Codes behind 2^32 bytes of the cache: the pages of the last sequence lie there."""
    n_kv, dim, page = 8, 128, 256
    n_pages = (1 << 32) // (n_kv * dim * page) + 6
    cache = bq.KvCache.empty(n_pages, n_kv, dim, page, dev)
    table = torch.tensor([[n_pages - 1, n_pages - 3]], dtype=torch.int32, device=dev)
    kv = 300
    K, V = _tokens(kv, n_kv, dim, "f16", 1, dev), _tokens(kv, n_kv, dim, "f16", 2, dev)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    bq.bpdq_kv_write(cache, table, ints([0]), ints([0, kv]), K, V)
    Q = torch.randn((3, 16, dim), generator=torch.Generator().manual_seed(5)).half().to(dev)
    out = bq.bpdq_kv_attention(cache, table, ints([kv]), ints([0, 3]), Q)
    seq = Sequences(dev, 1, n_kv, dim, page, kv, 1)
    seq.write([kv], K, V)
    assert torch.equal(out, _attend(seq, Q, [3], lse=False)[0]) or \
        torch.allclose(out.float(), _attend(seq, Q, [3], lse=False)[0].float(), atol=2e-3)      # another split of the table's room
    back, _ = bq.bpdq_kv_read(cache, table, ints([0]), ints([0, kv]), kv)
    assert torch.equal(back, bq.bpdq_kv_read(seq.cache, seq.table_d, ints([0]), ints([0, kv]), kv)[0])


def test_attention_refuses_tensors(dev):
    seq = Sequences(dev, 1, 2, 64, 64, 64, 1)
    Q = torch.zeros((1, 4, 64), dtype=torch.float16, device=dev)
    n, s = seq.ints([1]), seq.ints([0, 1])
    for bad in (lambda: bq.bpdq_kv_attention(seq.cache, seq.table_d, n, s, Q.float()),
                lambda: bq.bpdq_kv_attention(seq.cache, seq.table_d, n, s, Q[:, :3]),
                lambda: bq.bpdq_kv_attention(seq.cache, seq.table_d, n, s, Q[:, :, :32]),
                lambda: bq.bpdq_kv_attention(seq.cache, seq.table_d, n, s, Q, max_kv=65),
                lambda: bq.bpdq_kv_attention(seq.cache, seq.table_d, n, s, Q, window=-1),
                lambda: bq.bpdq_kv_attention(seq.cache, seq.table_d, n, s, Q, scale=float("nan")),
                lambda: bq.bpdq_kv_attention(seq.cache, seq.table_d, n, s, Q, out=Q.float()),
                lambda: bq.bpdq_kv_attention(seq.cache, seq.table_d, n, s, Q, lse=torch.zeros(4, device=dev)),
                lambda: bq.bpdq_kv_attention(seq.cache, seq.table_d, n, s, Q.cpu())):
        with pytest.raises(bq.BpdqError):
            bad()
    assert bq.bpdq_kv_attention(seq.cache, seq.table_d, n, seq.ints([0, 0]), Q[:0]).shape == (0, 4, 64)


# ------------------------------------------------------------------ streams and graphs

def test_a_step_on_another_stream_and_in_a_graph(dev):
    """Write, attention over a split cache and the product behind it, on a side stream and as a replayed graph: the eager result every
    time, with eager work between the replays."""
    n_kv, dim, n_q, kv = 2, 128, 8, 2000
    seq = Sequences(dev, 1, n_kv, dim, 64, kv + 1, 19)
    seq.write([kv], _tokens(kv, n_kv, dim, "bf16", 1, dev), _tokens(kv, n_kv, dim, "bf16", 2, dev))
    p, c = _on(*_layer(256, n_q * dim, 2, 64, 3), dev)
    K, V = _tokens(1, n_kv, dim, "bf16", 3, dev), _tokens(1, n_kv, dim, "bf16", 4, dev)
    Q = torch.randn((1, n_q, dim), generator=torch.Generator().manual_seed(5)).bfloat16().to(dev)
    table, pos, n, start = seq.table_d, seq.ints([kv]), seq.ints([kv + 1]), seq.ints([0, 1])
    ws = torch.empty(bq.bpdq_kv_attention_workspace_bytes(1, 1, kv + 1, n_q, n_kv, dim), dtype=torch.uint8, device=dev)
    assert ws.numel() > 0
    out, y = torch.empty_like(Q), torch.empty((1, 256), dtype=torch.bfloat16, device=dev)

    def step():
        bq.bpdq_kv_write(seq.cache, table, pos, start, K, V)
        bq.bpdq_kv_attention(seq.cache, table, n, start, Q, 1, kv + 1, out=out, ws=ws)
        bq.bpdq_linear(p, c, 64, out.view(1, -1), act="silu", Y=y)

    step()
    torch.cuda.synchronize()
    want, want_out = y.clone(), out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in range(4):
        y.zero_()
        out.zero_()
        ws.fill_(i)
        torch.randn((300, 300), device=dev).sum()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(out, want_out), i


def test_calls_allocate_nothing(dev):
    """With outputs and workspace given, a step allocates no device memory."""
    seq = Sequences(dev, 1, 1, 64, 64, 64, 1)
    x = _tokens(5, 1, 64, "f16", 1, dev)
    Q, out = torch.zeros((5, 2, 64), dtype=torch.float16, device=dev), torch.empty((5, 2, 64), dtype=torch.float16, device=dev)
    p, c = _on(*_layer(32, 128, 2, 32, 3), dev)
    y = torch.empty((5, 32), dtype=torch.float16, device=dev)
    table, pos, n, start = seq.table_d, seq.ints([0]), seq.ints([5]), seq.ints([0, 5])
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    bq.bpdq_kv_write(seq.cache, table, pos, start, x, x)
    bq.bpdq_kv_attention(seq.cache, table, n, start, Q, out=out)
    bq.bpdq_linear(p, c, 32, out.view(5, 128), Y=y)
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() == before


def test_the_example(dev):
    """The example's block, prompt and decoded tokens, against 64 bits, the attention's output apart from the residual.  Attention: a step of the
    cache is at most twice amax / 127 (a scale that grew), and with amax below 6 rms its rounding, redone once, has a standard deviation of
    2 * 6 / 127 / sqrt(12) * sqrt(1.25) = 3.1 % of V's, which attention averages as it averages V itself; q, k, v and the output are rounded to
    bfloat16, 2^-9 each, and K's rounding moves scores that are small here: below 4 %.  Block: 2^-9 of its norm for its own rounding
    and, of what it adds, the attention's 4 % and the product's rounding: 5 %."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_attention.py")
    spec = importlib.util.spec_from_file_location("serve_attention", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    for attention, whole, share in example.main(["--tokens", "150", "--decode", "20"]):
        assert attention < 0.04
        assert whole < 2.0 ** -9 + 0.05 * share
