"""The norm, rotary positions, the gated product and sampling on the GPU, through the binding, against the numpy oracle in 64 bits.

Tolerances.  u = 2^-11 (float16), 2^-8 (bfloat16) or 2^-24 (float32) is the largest relative error of one rounding to the type, e = 2^-24 that of
fp32, z the least magnitude with all its bits (2^-14, else 2^-126: below it, roundings cost u z at most).
Norm: the sum is off by e of itself, and so is their root mean square; its reciprocal, offset + weight, two products: 6 e in all, 8 with room, and u.
Codes: y / scale is off by those 8 e, 2 e of the scale and 2 e of the quotient, times up to 127.
Rotary: the fraction of a turn is at most 1/2 and rounded to fp32, 2^-26 of a turn or 1.6 e; sine and cosine of a library good to 4 e; mscale e; two
products and a sum 2 e: below 10 e of mscale (|a| + |b|), and u; and the fp64 angle, 2^-51 of itself.
Gated: both projections as in the product's tests, (w + (d + 16) e) S each, w = 2^-11 the rounding of a weight to fp16; the activation's slope is
below 1.13, and its own error 2^-16 of it and 2^-21 of its argument.  Over all values: a projection's error is a sum of independent terms w |W| |x| at most,
so below w times the root of their sum of squares.
Sampling: a weight is off by half a unit of 2^-43 of the largest, so a running sum by n 2^-44 and the share of the total that it is compared with by as
much: tokens are equal unless they are within n 2^-43 (the oracle says how near they came); prob 4 e.
"""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as do
from paper_2602_04163_amd import binding as bq

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
LEAST = {"f32": 2.0 ** -126, "f16": 2.0 ** -14, "bf16": 2.0 ** -126}
E, W16 = 2.0 ** -24, 2.0 ** -11
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    bq.load()
    return torch.device("cuda:0")


def _np(t):
    return t.detach().double().cpu().numpy()


def _ints(v, dev):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def _inside(x, ld, at=0):
    """x with rows ld apart, from the at-th element of its storage on."""
    n = x.shape[0]
    big = torch.full((n * ld + at + 8,), 7, dtype=x.dtype, device=x.device)
    view = big[at:at + n * ld].view(n, ld)[:, :x[0].numel()].unflatten(1, x.shape[1:])
    view.copy_(x)
    return view


# ------------------------------------------------------------------ norm

def _norm_inputs(n, d, kind, wide, seed, dev, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    loud = torch.exp(0.5 * torch.randn(d, generator=g))
    x = (scale * torch.randn((n, d), generator=g) * loud).to(TYPES[kind])
    r = None if wide is None else (3 * scale * torch.randn((n, d), generator=g)).to(TYPES[wide])
    w = (1 + 0.3 * torch.randn(d, generator=g)).to(TYPES[kind])
    return x.to(dev), None if r is None else r.to(dev), w.to(dev)


def _check_norm(y, s, x, r, w, kind, wide, offset=0.0, eps=1e-6):
    want_s, want = do.rms_norm(_np(x), None if r is None else _np(r), None if w is None else _np(w), offset, eps)
    tol = (8 * E + U[kind]) * np.abs(want) + U[kind] * LEAST[kind]
    assert (np.abs(_np(y) - want) <= tol).all(), np.max(np.abs(_np(y) - want) / tol)
    if r is not None:
        tol = U[wide] * (1 + E) * np.abs(want_s) + E * np.abs(want_s) + U[wide] * LEAST[wide]
        assert s.dtype is TYPES[wide] and (np.abs(_np(s) - want_s) <= tol).all()
    return want


NORMS = [(1, 1, "f32", None), (3, 7, "bf16", "bf16"), (5, 8, "f16", "f32"), (2, 63, "f32", "f32"), (4, 64, "bf16", None), (9, 128, "f16", "f16"),
         (7, 511, "bf16", "f32"), (6, 513, "f16", None), (33, 1000, "f32", "f32"), (17, 1024, "bf16", "bf16"), (16, 3584, "bf16", "f32"),
         (300, 3584, "f16", "f16"), (5, 3583, "bf16", "bf16"), (3, 8192, "bf16", "f32"), (2, 8200, "f32", None), (2, 16383, "f16", "f32"),
         (3, 18944, "f16", None), (2, 29568, "bf16", "bf16"), (1, 32776, "f32", "f32"), (2, 65535, "bf16", "f32"), (1, 65536, "f16", "f16"),
         (5000, 96, "bf16", "bf16"), (1500, 2048, "f32", "f32"), (1100, 5000, "bf16", "f32"), (700, 9000, "f16", "f16")]


@pytest.mark.parametrize("n,d,kind,wide", NORMS)
def test_norm(dev, n, d, kind, wide):
    print(f"norm {n} x {d} {kind} + {wide}", flush=True)
    x, r, w = _norm_inputs(n, d, kind, wide, n + d, dev)
    y, s = bq.bpdq_rms_norm(x, w, residual=r)
    _check_norm(y, s, x, r, w, kind, wide)
    again, _ = bq.bpdq_rms_norm(x, w, residual=r)
    assert torch.equal(y, again)


@pytest.mark.parametrize("kind,wide,pad,at", [("bf16", "bf16", 8, 0), ("bf16", "f32", 1, 0), ("f16", "f16", 8, 1), ("f32", "f32", 3, 1), ("f16", "f32", 4, 2)])
def test_norm_strides(dev, kind, wide, pad, at):
    """Rows apart and odd addresses; what lies between the rows stays."""
    for d in (40, 520, 4097):
        x, r, w = _norm_inputs(6, d, kind, wide, d, dev)
        y, s = _inside(torch.zeros_like(x), d + pad, at), _inside(torch.zeros_like(r), d + pad, at)
        bq.bpdq_rms_norm(_inside(x, d + pad, at), w, residual=_inside(r, d + pad, at), S=s, Y=y, offset=1.0)
        _check_norm(y, s, x, r, w, kind, wide, offset=1.0)
        for t in (y, s):
            assert (t.as_strided((6, pad), (d + pad, 1), at + d) == 7).all()


def test_norm_in_place(dev):
    """The sum over the residual or over X, Y over X."""
    x, r, w = _norm_inputs(40, 3584, "bf16", "bf16", 1, dev)
    y, s = bq.bpdq_rms_norm(x, w, residual=r)
    r2 = r.clone()
    y2, s2 = bq.bpdq_rms_norm(x, w, residual=r2, S=r2)
    assert s2 is r2 and torch.equal(y2, y) and torch.equal(r2, s)
    x2, r2 = x.clone(), r.clone()
    bq.bpdq_rms_norm(x2, w, residual=r2, S=r2, Y=x2)
    assert torch.equal(x2, y) and torch.equal(r2, s)
    x2 = x.clone()
    bq.bpdq_rms_norm(x2, w, residual=r, S=x2, Y=torch.empty_like(x))
    assert torch.equal(x2, s)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1e-30, 1e30])
def test_norm_magnitudes(dev, kind, scale):
    """Squares that leave fp32."""
    for d in (200, 4000):
        x, r, w = _norm_inputs(4, d, kind, kind, d, dev, scale)
        y, s = bq.bpdq_rms_norm(x, w, residual=r, eps=1e-37)
        _check_norm(y, s, x, r, w, kind, kind, eps=float(np.float32(1e-37)))
    x = torch.zeros((3, 300), dtype=TYPES[kind], device=dev)
    assert (bq.bpdq_rms_norm(x)[0] == 0).all()


def test_norm_without_weight_and_without_rows(dev):
    x, _, _ = _norm_inputs(3, 100, "f32", None, 5, dev)
    _check_norm(bq.bpdq_rms_norm(x)[0], None, x, None, None, "f32", None)
    y, s = bq.bpdq_rms_norm(torch.empty((0, 64), device=dev))
    assert y.shape == (0, 64) and s is None


def test_norm_keeps_what_is_no_number_in_its_row(dev):
    for d in (100, 3000):
        x, r, w = _norm_inputs(6, d, "bf16", "f32", 3, dev)
        clean, _ = bq.bpdq_rms_norm(x, w, residual=r)
        x[1, 7], r[3, d - 1] = NAN, INF
        y, s = bq.bpdq_rms_norm(x, w, residual=r)
        assert y[1].isnan().all() and y[3, d - 1].isnan() and (y[3, :d - 1] == 0).all()
        for i in (0, 2, 4, 5):
            assert torch.equal(y[i], clean[i])
        codes, scales, _ = bq.bpdq_rms_norm_q8(x, w, residual=r)
        assert scales.isnan()[:, 0].tolist() == [False, True, False, True, False, False]


@pytest.mark.parametrize("n,d,group,kind,wide", [
    (1, 1, 0, "f32", None), (5, 32, 32, "bf16", "bf16"), (3, 96, 32, "f16", None), (9, 500, 0, "bf16", "f32"), (4, 512, 256, "f32", "f32"),
    (6, 640, 64, "f16", "f16"), (3, 1023, 0, "f32", None), (7, 3584, 128, "bf16", "f32"), (2, 8320, 64, "bf16", None), (3, 18944, 0, "f16", None),
    (3, 18944, 128, "f16", "f32"), (2, 29568, 32, "bf16", "bf16"), (1, 65536, 256, "f16", None), (1, 65531, 0, "bf16", None),
    (2000, 256, 64, "bf16", "bf16"), (600, 4096, 0, "f32", "f32")])
def test_norm_codes(dev, n, d, group, kind, wide):
    print(f"norm codes {n} x {d} / {group} {kind} + {wide}", flush=True)
    x, r, w = _norm_inputs(n, d, kind, wide, n + d + 1, dev)
    codes, scales, s = bq.bpdq_rms_norm_q8(x, w, residual=r, group=group)
    _, want = do.rms_norm(_np(x), None if r is None else _np(r), _np(w))
    step = do.scales(want, group)
    assert scales.shape == step.shape and (np.abs(_np(scales) - step) <= 12 * E * step).all()
    exact = want.reshape(n, -1, group or d) / step[:, :, None]
    got = _np(codes).reshape(exact.shape)
    assert (np.abs(got - exact) <= 0.5 + 127 * 12 * E).all() and (np.abs(got).max(2) == 127).all()
    if r is not None:
        assert torch.equal(s, bq.bpdq_rms_norm(x, w, residual=r)[1])


def test_norm_codes_strides(dev):
    x, _, w = _norm_inputs(5, 96, "bf16", None, 9, dev)
    codes, scales, _ = bq.bpdq_rms_norm_q8(x, w, group=32)
    for pad, at in ((8, 0), (1, 0), (8, 3)):
        into = _inside(torch.zeros((5, 96), dtype=torch.int8, device=dev), 96 + pad, at)
        bq.bpdq_rms_norm_q8(x, w, group=32, codes=into)
        assert torch.equal(into, codes) and (into.as_strided((5, pad), (96 + pad, 1), at + 96) == 7).all()
    zero, scales, _ = bq.bpdq_rms_norm_q8(torch.zeros_like(x), w)
    assert (zero == 0).all() and (_np(scales) == np.float32(2.0 ** -96) * (np.float32(1) / np.float32(127))).all()


# ------------------------------------------------------------------ rotary positions

def _positions(pos, start):
    return np.concatenate([np.arange(p, p + b - a) for p, a, b in zip(pos, start, start[1:])] or [np.zeros(0)]).astype(np.float64)


def _check_turned(got, x, at, freq, layout, mscale, inverse, kind):
    want = do.rotary(_np(x), at, freq, layout, mscale, inverse)
    half = len(freq)
    size = np.abs(_np(x))
    i = np.arange(half)
    a, b = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
    both = abs(mscale) * (size[:, :, a] + size[:, :, b])
    far = 2.0 ** -51 * np.abs(np.outer(at, freq))[:, None]
    tol = U[kind] * np.abs(want) + U[kind] * LEAST[kind]
    tol[:, :, a] += (10 * E + far) * both
    tol[:, :, b] += (10 * E + far) * both
    tol[:, :, 2 * half:] = 0
    assert (np.abs(_np(got) - want) <= tol).all(), np.max(np.abs(_np(got) - want) - tol)


@pytest.mark.parametrize("counts,pos,n_q,n_kv,dim,rot,layout,kind", [
    ([1], [0], 1, 1, 2, 2, "half", "f32"), ([1], [1000], 28, 4, 128, 128, "half", "bf16"), ([1] * 16, range(0, 1600, 100), 28, 4, 128, 128, "half", "f16"),
    ([5, 0, 1, 17], [3, 9, 0, 1 << 20], 15, 5, 64, 32, "interleaved", "bf16"), ([300], [120000], 64, 8, 128, 64, "half", "f16"),
    ([7, 9], [1 << 30, (1 << 31) - 9], 6, 3, 80, 80, "half", "f32"), ([33], [5], 4, 0, 256, 256, "interleaved", "f16"),
    ([4, 4], [0, 1], 3, 1, 66, 22, "half", "bf16"), ([4, 4], [0, 1], 3, 1, 66, 22, "interleaved", "f32"), ([2], [11], 2, 2, 512, 510, "half", "f16"),
    ([2], [11], 2, 2, 512, 512, "interleaved", "f32"), ([64] * 20, range(20), 8, 2, 64, 64, "half", "bf16"), ([3000], [0], 2, 1, 96, 96, "half", "f16"),
    ([3], [4], 200, 100, 16, 6, "interleaved", "bf16")])
def test_rotary(dev, counts, pos, n_q, n_kv, dim, rot, layout, kind):
    print(f"rotary {counts} {n_q}/{n_kv} x {dim} rot {rot} {layout} {kind}", flush=True)
    pos, start = list(pos), [0] + np.cumsum(counts).tolist()
    n = start[-1]
    g = torch.Generator().manual_seed(n + dim)
    q = torch.randn((n, n_q, dim), generator=g).to(TYPES[kind]).to(dev)
    k = torch.randn((n, n_kv, dim), generator=g).to(TYPES[kind]).to(dev) if n_kv else None
    freq, _ = do.rotary_frequencies(rot, 1e4)
    f, p, s = torch.tensor(freq, device=dev), _ints(pos, dev), _ints(start, dev)
    at = _positions(pos, start)
    for mscale, inverse in ((1.0, False), (1.25, True)):
        q2, k2 = bq.bpdq_rotary(f, p, s, q, k, max_tok=max(counts), layout=layout, mscale=mscale, inverse=inverse)
        _check_turned(q2, q, at, freq, layout, mscale, inverse, kind)
        if n_kv:
            _check_turned(k2, k, at, freq, layout, mscale, inverse, kind)
    # in place, and with nothing said about the largest count
    q2, k2 = bq.bpdq_rotary(f, p, s, q, k, layout=layout)
    q3, k3 = q.clone(), None if k is None else k.clone()
    bq.bpdq_rotary(f, p, s, q3, k3, max_tok=max(counts), layout=layout, Q_out=q3, K_out=k3)
    assert torch.equal(q2, q3) and (k is None or torch.equal(k2, k3))


@pytest.mark.parametrize("pad,at,rot", [(0, 0, 64), (8, 0, 32), (1, 0, 64), (8, 1, 64), (0, 0, 30)])
def test_rotary_strides(dev, pad, at, rot):
    """Q and K of one product side by side, rows apart, odd addresses, pairs that are no whole vectors: the same results to the bit."""
    g = torch.Generator().manual_seed(1)
    qkv = torch.randn((9, 8 * 64), generator=g).half().to(dev)
    f, p, s = torch.tensor(do.rotary_frequencies(rot)[0], device=dev), _ints([100, 5], dev), _ints([0, 4, 9], dev)
    q, k = qkv[:, :256].unflatten(1, (4, 64)), qkv[:, 256:384].unflatten(1, (2, 64))
    for layout in ("half", "interleaved"):
        q0, k0 = bq.bpdq_rotary(f, p, s, q.contiguous(), k.contiguous(), layout=layout)
        moved = _inside(qkv, 512 + pad, at)
        mq, mk = moved[:, :256].unflatten(1, (4, 64)), moved[:, 256:384].unflatten(1, (2, 64))
        out = _inside(torch.zeros_like(q), 256 + pad, at)
        q1, k1 = bq.bpdq_rotary(f, p, s, mq, mk, layout=layout, Q_out=out)
        assert torch.equal(q1, q0) and torch.equal(k1, k0)
        bq.bpdq_rotary(f, p, s, mq, mk, layout=layout, Q_out=mq, K_out=mk)
        assert torch.equal(mq, q0) and torch.equal(mk, k0) and torch.equal(moved[:, 384:], qkv[:, 384:])


def test_rotary_leaves_rows_alone(dev):
    """Rows that no sequence names, of a sequence with a negative position, beyond max_tok, beyond n_tok."""
    f, q = torch.ones(8, dtype=torch.float64, device=dev), torch.randn((12, 2, 16), device=dev)
    out = torch.full_like(q, 5)
    bq.bpdq_rotary(f, _ints([4, -1, 7], dev), _ints([1, 4, 6, 40], dev), q, Q_out=out, max_tok=2)
    turned, _ = bq.bpdq_rotary(f, _ints([3, 5], dev), _ints([0, 4, 12], dev), q)        # rows 1, 2 and 6, 7 at the same positions
    assert [i for i in range(12) if (out[i] == 5).all()] == [0, 3, 4, 5, 8, 9, 10, 11]
    assert torch.equal(out[1:3], turned[1:3]) and torch.equal(out[6:8], turned[6:8])
    before = out.clone()
    bq.bpdq_rotary(f, _ints([0, 0], dev), _ints([-3, 0, 0], dev), q, Q_out=out)
    bq.bpdq_rotary(f, _ints([], dev), _ints([0], dev), q, Q_out=out)
    assert torch.equal(out, before)


# ------------------------------------------------------------------ the gated product

def _layer(rows, d_in, bits, group, seed):
    g = np.random.default_rng(seed)
    planes = g.integers(0, 1 << 32, (bits, rows, d_in // 32), dtype=np.uint32)
    coefs = (g.standard_normal((bits + 1, rows, d_in // group)) * (1.5 / d_in ** 0.5)).astype(np.float16)
    return planes, coefs


def _on(planes, coefs, dev):
    return torch.from_numpy(planes.view(np.int32)).to(dev), torch.from_numpy(coefs).to(dev)


def _check_gated(y, planes, coefs, group, x, bias, name, kind):
    d_in = x.shape[1]
    want, (gate, up), (size_g, size_u), (root_g, root_u) = do.gated(planes, coefs, group, _np(x), None if bias is None else _np(bias), name)
    u, act = U[kind], do.so.act(gate, name)
    off_g = 1.13 * (W16 + (d_in + 16) * E) * size_g + 2.0 ** -16 * np.abs(act) * (1 + np.abs(gate) / 32) + 2.0 ** -24
    off_u = (W16 + (d_in + 16) * E) * size_u + 2.0 ** -24
    tol = off_g * np.abs(up) + off_u * np.abs(act) + off_g * off_u + u * np.abs(want) + u * LEAST[kind]
    got = _np(y)
    assert (np.abs(got - want) <= tol).all(), np.max(np.abs(got - want) / tol)
    parts = np.sqrt((1.13 * W16 * root_g * up) ** 2 + (W16 * root_u * act) ** 2)
    most = u * np.linalg.norm(want) + np.linalg.norm(parts) + 2.0 ** -15 * np.linalg.norm(want) + 2.0 ** -24 * np.sqrt(want.size)
    assert np.linalg.norm(got - want) <= most, np.linalg.norm(got - want) / most


GATED = [(2, 128, 48, 512, 1, "bf16", "silu", False), (2, 64, 33, 640, 1, "f16", "gelu", True), (1, 32, 1, 32, 2, "f16", "none", True),
         (3, 32, 7, 96, 3, "bf16", "relu", False), (4, 64, 130, 1088, 5, "f16", "silu", True), (2, 96, 65, 288, 15, "bf16", "gelu_tanh", True),
         (3, 128, 64, 4096, 16, "f16", "silu", False), (1, 256, 257, 768, 17, "bf16", "silu", True), (2, 32, 31, 8224, 31, "f16", "relu", False),
         (4, 32, 100, 2080, 32, "bf16", "none", True), (2, 128, 300, 1152, 33, "f16", "gelu", False), (3, 64, 64, 64, 64, "bf16", "none", False),
         (2, 64, 201, 1984, 65, "bf16", "silu", True), (3, 256, 513, 1280, 127, "f16", "gelu_tanh", True), (2, 128, 128, 512, 128, "bf16", "silu", True),
         (1, 32, 255, 416, 129, "f16", "none", False), (4, 128, 383, 640, 200, "bf16", "relu", True), (2, 128, 513, 2176, 257, "f16", "silu", False)]


@pytest.mark.parametrize("bits,group,f,d_in,n,kind,name,bias", GATED)
def test_gated(dev, bits, group, f, d_in, n, kind, name, bias):
    print(f"gated k={bits} g={group} 2x{f}x{d_in} n={n} {kind} {name}", flush=True)
    planes, coefs = _layer(2 * f, d_in, bits, group, f + d_in + n)
    g = torch.Generator().manual_seed(n)
    x = (torch.randn((n, d_in), generator=g) * torch.exp(0.5 * torch.randn(d_in, generator=g))).to(TYPES[kind]).to(dev)
    b = torch.randn(2 * f, generator=g).to(TYPES[kind]).to(dev) if bias else None
    p, c = _on(planes, coefs, dev)
    y = bq.bpdq_gated_linear(p, c, group, x, bias=b, act=name)
    _check_gated(y, planes, coefs, group, x, b, name, kind)
    assert torch.equal(y, bq.bpdq_gated_linear(p, c, group, x, bias=b, act=name))


# tokens, columns and pairs of rows at which each of the product's kernels is chosen (few tokens with 1, 2, 3, 5 and 8 row tiles, twice 16 tokens with
# 2, 3 and 5, tiles of 128 x 64, 128 x 128, 256 x 128 and 256 x 256): tests/test_gated_kernels.py has their rows
@pytest.mark.parametrize("n,d_in,f", [(1, 256, 1000), (65, 256, 1550), (65, 256, 2050), (700, 256, 260), (1500, 256, 65), (513, 256, 65), (257, 256, 260),
                                      (513, 256, 500), (257, 1024, 2500), (300, 512, 4100), (1025, 256, 2500), (1025, 256, 4099)])
@pytest.mark.parametrize("bits,group,kind", [(1, 128, "bf16"), (2, 64, "f16"), (3, 32, "bf16"), (4, 128, "f16"), (2, 0, "bf16")])
def test_gated_kernels(dev, n, d_in, f, bits, group, kind):
    """With groups of four words, of two and of one; with one word more to a row (group 0), so that rows are not 16 bytes and the last columns
    end inside a tile."""
    if group == 0:
        d_in, group = d_in + 32, (96 if (d_in + 32) % 96 == 0 else 32)
    print(f"gated kernels k={bits} g={group} 2x{f}x{d_in} n={n} {kind}", flush=True)
    planes, coefs = _layer(2 * f, d_in, bits, group, n)
    g = torch.Generator().manual_seed(n)
    x = (torch.randn((n, d_in), generator=g) * torch.exp(0.5 * torch.randn(d_in, generator=g))).to(TYPES[kind]).to(dev)
    b = torch.randn(2 * f, generator=g).to(TYPES[kind]).to(dev)
    p, c = _on(planes, coefs, dev)
    _check_gated(bq.bpdq_gated_linear(p, c, group, x, bias=b), planes, coefs, group, x, b, "silu", kind)


# columns and groups for which each form of the one-token kernel is chosen: one, two or four words to a lane, consecutive (sharing one group, two, four)
# and strided; below and above 256 rows of work-groups
@pytest.mark.parametrize("d_in,group", [(32, 32), (2048, 64), (2080, 32), (4096, 128), (4096, 32), (3584, 128), (4160, 32), (5120, 64), (8192, 128), (8192, 64),
                                        (8192, 32), (8160, 96), (6176, 32), (8224, 32)])
@pytest.mark.parametrize("bits,kind,f,bias", [(1, "f16", 300, True), (2, "bf16", 5000, False), (3, "f16", 17, False), (4, "bf16", 4100, True)])
def test_gated_token(dev, d_in, group, bits, kind, f, bias):
    print(f"gated token k={bits} g={group} 2x{f}x{d_in} {kind}", flush=True)
    planes, coefs = _layer(2 * f, d_in, bits, group, d_in + f)
    g = torch.Generator().manual_seed(d_in)
    x = (torch.randn((1, d_in), generator=g) * torch.exp(0.5 * torch.randn(d_in, generator=g))).to(TYPES[kind]).to(dev)
    b = torch.randn(2 * f, generator=g).to(TYPES[kind]).to(dev) if bias else None
    p, c = _on(planes, coefs, dev)
    y = bq.bpdq_gated_linear(p, c, group, x, bias=b)
    _check_gated(y, planes, coefs, group, x, b, "silu", kind)
    into = _inside(torch.zeros((1, f), dtype=x.dtype, device=dev), f + 3, 1)
    bq.bpdq_gated_linear(p, c, group, _inside(x, d_in + 1, 1), bias=b, Y=into)
    assert torch.equal(into, y)


def test_gated_token_magnitudes(dev):
    """Sums of the largest values of the type, with and without an infinity."""
    planes, coefs = _layer(2 * 40, 256, 2, 64, 7)
    p, c = _on(planes, coefs * np.float16(2.0 ** -6), dev)
    x = torch.full((1, 256), 2.0 ** 127, dtype=torch.bfloat16, device=dev)
    want, (gate, up), _, _ = do.gated(planes, coefs * np.float16(2.0 ** -6), 64, _np(x), None, "none")
    assert np.isfinite(want).all() and np.abs(gate).max() > 2.0 ** 120
    y = bq.bpdq_gated_linear(p, c, 64, x, act="relu")
    assert (_np(y)[np.abs(want) > 2.0 ** 129] != 0).any() and not y.isnan().any()
    x[0, 3] = INF
    assert not bq.bpdq_gated_linear(p, c, 64, x, act="none").isfinite().all()


@pytest.mark.parametrize("n", [3, 40])
def test_gated_strides_and_infinities(dev, n):
    planes, coefs = _layer(2 * 70, 320, 2, 64, 5)
    p, c = _on(planes, coefs, dev)
    x = torch.randn((n, 320), generator=torch.Generator().manual_seed(2)).bfloat16().to(dev)
    want = bq.bpdq_gated_linear(p, c, 64, x)
    for pad, at in ((8, 0), (1, 0), (8, 1)):
        y = _inside(torch.zeros_like(want), 70 + pad, at)
        bq.bpdq_gated_linear(p, c, 64, _inside(x, 320 + pad, at), Y=y)
        assert torch.equal(y, want) and (y.as_strided((n, pad), (70 + pad, 1), at + 70) == 7).all()
    x[1, 17], x[2, 5] = NAN, 3e38
    y = bq.bpdq_gated_linear(p, c, 64, x)
    assert y[1].isnan().all()
    for i in [0] + list(range(3, n)):
        assert torch.equal(y[i], want[i])
    assert bq.bpdq_gated_linear(p, c, 64, x[:0]).shape == (0, 70)


def test_gated_is_two_products(dev):
    """Layers that share one input, through the sweep in one call: the gated product is act(gate) * up of the two by themselves."""
    g = torch.Generator(device=dev).manual_seed(3)
    W, X = 0.02 * torch.randn((2 * 96, 256), generator=g, device=dev), torch.randn((512, 256), generator=g, device=dev)
    H = torch.zeros((256, 256), device=dev)
    bq.bpdq_hessian_accumulate(X, H)
    U_, dead, _ = bq.bpdq_prepare(H)
    out = bq.bpdq_quantize_layers(W, [96, 192], U_, dead, bq.make_params(2, 64, 64, 2, coef_fp16=True))
    planes, coefs = out["planes"], bq.bpdq_coefs_to_fp16(out["coefs"])
    x = X[:50].half()
    gate, up = [bq.bpdq_linear(planes[:, at:at + 96].contiguous(), coefs[:, at:at + 96].contiguous(), 64, x, act=a) for at, a in ((0, "silu"), (96, "none"))]
    y = bq.bpdq_gated_linear(planes, coefs, 64, x)
    # two roundings of the factors more, whose sums may be ordered otherwise
    assert ((y.float() - gate.float() * up.float()).abs() <= 4 * U["f16"] * (gate.float() * up.float()).abs() + 2.0 ** -14).all()


# ------------------------------------------------------------------ sampling

def _check_sample(x, u, t=None, k=None, p=None, m=None, dev=None, whole=False):
    """x (n, vocab) on the GPU; every row against the oracle.  whole, or a row of one value, or with plus infinities: the weights that
    count are 1 and 0, so sums and shares (24 bits times 20) are exact in fp64 too, and borders are borders."""
    n, vocab = x.shape
    on = lambda v, kind: None if v is None else torch.tensor(v, dtype=kind, device=dev)  # noqa: E731
    t_, k_, p_, m_, u_ = on(t, torch.float32), on(k, torch.int32), on(p, torch.float32), on(m, torch.float32), on(u, torch.float32)
    token, prob = bq.bpdq_sample(x, u_, temperature=t_, top_k=k_, top_p=p_, min_p=m_, want_prob=True)
    assert torch.equal(token, bq.bpdq_sample(x, u_, temperature=t_, top_k=k_, top_p=p_, min_p=m_))
    host, got, pr = _np(x), token.tolist(), _np(prob)
    one = lambda v, i, default: default if v is None else float(v[i])  # noqa: E731
    unsure = 0
    for i in range(n):
        want, q, _, margin = do.sample(np.where(np.isnan(host[i]), -np.inf, host[i]), one(u_, i, 0), one(t_, i, 1.0), int(one(k_, i, 0)), one(p_, i, 1.0),
                                       one(m_, i, 0.0))
        there = host[i][host[i] > -np.inf]
        if margin <= vocab * 2.0 ** -43 and not (whole or there.min() == there.max() or there.max() == np.inf):
            unsure += 1
            continue
        assert got[i] == want, (i, got[i], want, margin)
        assert abs(pr[i] - q) <= 4 * E * q + vocab * 2.0 ** -43
    assert unsure == 0
    return got


def _logits(n, vocab, kind, seed, dev, spread=2.0, masked=0.0):
    g = torch.Generator().manual_seed(seed)
    x = spread * torch.randn((n, vocab), generator=g)
    x.scatter_add_(1, torch.randint(0, vocab, (n, 12), generator=g), 9 * torch.rand((n, 12), generator=g))
    if masked:
        hide = torch.rand((n, vocab), generator=g) < masked
        hide[:, vocab // 2] = False
        x = x.masked_fill(hide, -INF)
    u = torch.rand(n, generator=g).tolist()
    return x.to(TYPES[kind]).to(dev), u


@pytest.mark.parametrize("n,vocab,kind,masked", [(1, 1, "f32", 0), (2, 2, "bf16", 0), (7, 5, "f16", 0), (12, 63, "f32", 0), (12, 1000, "bf16", 0.9), (24, 1025, "f16", 0),
                                                 (24, 4099, "f32", 0.99), (12, 20000, "bf16", 0), (6, 32003, "f16", 0.5), (6, 152064, "f32", 0), (2, 262144, "bf16", 0),
                                                 (300, 77, "f32", 0.5)])
def test_sample(dev, n, vocab, kind, masked):
    """Every filter alone, together, off, and greedy rows, by row in one call; and the calls that leave an argument out."""
    print(f"sample {n} x {vocab} {kind}", flush=True)
    x, u = _logits(n, vocab, kind, vocab, dev, masked=masked)
    row = np.arange(n)
    t = np.where(row % 7 == 3, 0.0, 0.6 + 0.2 * (row % 4))
    k = np.where(row % 3 == 0, 0, 1 + (row * 7) % 60)
    p = np.where(row % 4 == 0, 1.0, 0.5 + 0.1 * (row % 5))
    m = np.where(row % 5 < 3, 0.0, 0.05 * (row % 5))
    _check_sample(x, u, t, k, p, m, dev)
    _check_sample(x, u, dev=dev)
    _check_sample(x, u, t + 0.1, None, p, None, dev)
    _check_sample(x, u, None, k, None, None, dev)
    _check_sample(x, u, t, None, None, m, dev)


@pytest.mark.parametrize("kind,spread", [("f32", 0.02), ("bf16", 0.3), ("f16", 20.0), ("f32", 1e4), ("f32", 1e-6)])
def test_sample_spreads(dev, kind, spread):
    """Flat rows, where thousands of tokens are kept and thousands share a value, and steep ones."""
    x, u = _logits(16, 30011, kind, 4, dev, spread)
    if spread < 1:
        x -= x.max(1, keepdim=True).values / 2 if spread > 1e-3 else 0
    row = np.arange(16)
    _check_sample(x, u, np.full(16, 1.0), np.where(row % 2 == 0, 0, 500 * row), np.where(row % 3 == 0, 1.0, 0.1 + 0.05 * row), None, dev)
    _check_sample(x, u, np.full(16, 30.0), np.where(row % 2 == 0, 0, 29000), np.where(row % 2 == 1, 1.0, 0.97), np.full(16, 0.2), dev)


def test_sample_ties(dev):
    """Equal values: the lowest index first, to the last one that is kept."""
    n, vocab = 40, 5000
    x = torch.zeros((n, vocab), device=dev)
    u = [(i + 0.5) / n for i in range(n)]
    assert _check_sample(x, u, dev=dev) == [int(v * vocab) for v in u]
    assert _check_sample(x, u, k=[1000] * n, dev=dev) == [int(v * 1000) for v in u]
    for i, v in enumerate(bq.bpdq_sample(x, torch.tensor(u, device=dev), top_p=torch.full((n,), 0.5, device=dev)).tolist()):
        assert v == int(u[i] * 2500)                     # half of them to the token: sums of equal weights are exact
    x[:, ::2] = 1.0                                       # 2500 of them: two keys
    _check_sample(x, u, k=[2500 + 10 * i for i in range(n)], dev=dev)
    _check_sample(x, u, k=[2400] * n, p=[0.3 + 0.01 * i for i in range(n)], dev=dev, whole=True)
    x[:, :] = -0.0
    x[:, 1::2] = 0.0                                      # one value
    assert _check_sample(x, u, k=[3] * n, dev=dev) == [int(v * 3) for v in u]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_sample_orders(dev, kind):
    """Rows in rising and falling order, where all of the largest values lie in a few turns, and rows whose border's bin holds 65 to 4000 values."""
    n, vocab = 8, 40000
    g = torch.Generator().manual_seed(9)
    x = torch.randn((n, vocab), generator=g).sort(1).values
    x[1::2] = x[1::2].flip(1)
    x[4:] = 3.0 + (x[4:] * torch.tensor([0.003, 0.01, 0.03, 0.2])[:, None])
    x[4:, 77] = 12.0
    x, u = x.to(TYPES[kind]).to(dev), torch.rand(n, generator=g).tolist()
    for k in (1, 7, 19, 20, 39, 40, 100, 129, 600, 3000, 39999):
        _check_sample(x, u, k=[k] * n, dev=dev)
        _check_sample(x, u, t=[0.7] * n, k=[k] * n, p=[0.6 + 0.04 * i for i in range(n)], dev=dev)
    for p in (0.01, 0.2, 0.5, 0.99):
        _check_sample(x, u, p=[p] * n, m=[0.0, 0.3] * (n // 2), dev=dev)


def test_sample_steep(dev):
    """Temperatures at the ends of fp32 with min-p, on values that differ by next to nothing."""
    x = torch.zeros((4, 3000), device=dev)
    x[:, 5::7] = -1e-45
    x[2:, 6::7] = -1e-38
    u = [0.3, 0.8, 0.3, 0.8]
    _check_sample(x, u, t=[1e-40, 1e-44, 1e-40, 1e-38], m=[0.5, 0.01, 0.5, 0.3], dev=dev)
    _check_sample(x, u, t=[3e38, 1e30, INF, 1e-45], m=[0.999, 0.01, 0.5, 0.3], dev=dev)


def test_sample_what_is_no_number(dev):
    x = torch.randn((10, 3000), generator=torch.Generator().manual_seed(1)).to(dev)
    x[0] = -INF
    x[1] = NAN
    x[2, ::2], x[2, 1::2] = NAN, -INF
    x[2, 1234] = -3e38
    x[3, 7] = NAN
    x[4, [5, 2000]] = INF
    x[5] = INF
    x[6, :] = 3.4e38
    x[7, ::3] = -3.4e38
    u = [0.6] * 10
    got = _check_sample(x, u, dev=dev)
    assert got[:3] == [-1, -1, 1234] and got[4] == 2000 and got[5] == 1800
    for kw in (dict(k=[4] * 10), dict(p=[0.9] * 10), dict(k=[100] * 10, p=[0.5] * 10, m=[0.1] * 10), dict(t=[0.0] * 10), dict(t=[1e-40] * 10)):
        got = _check_sample(x, u, dev=dev, **kw)
        assert got[:3] == [-1, -1, 1234]


def test_sample_borders_of_its_arguments(dev):
    x, _ = _logits(8, 4000, "f32", 6, dev)
    best = x.argmax(1).tolist()
    u = [0.37] * 8
    # asked for the largest; one token left by each filter
    assert _check_sample(x, u, t=[0.0, -1.0, NAN, -INF, 0.0, -0.0, 0.0, 0.0], dev=dev) == best
    assert _check_sample(x, u, k=[1] * 8, dev=dev) == best
    assert _check_sample(x, u, p=[0.0, -1.0, -INF, 0.0, 1e-9, 1e-40, 0.0, 0.0], dev=dev) == best
    assert _check_sample(x, u, m=[1.0, 2.0, INF, 1.0, 1.0, 1.0, 1.0, 1.0], dev=dev) == best
    # filters that are off
    free = _check_sample(x, u, dev=dev)
    assert free == _check_sample(x, u, k=[0, -1, 4000, 4001, 1 << 30, -5, 0, 0], p=[1.0, 1.5, INF, NAN, 1.0, 1.0, 1.0, 1.0], m=[0.0, -1.0, NAN, -INF, 0.0, 0.0, 0.0, 0.0],
                                 dev=dev)
    flat = _check_sample(x, u, t=[INF] * 8, dev=dev)
    assert flat == [int(np.float32(0.37) * 4000.0)] * 8
    # u at and beyond its ends
    token = bq.bpdq_sample(x, torch.tensor([0.0, -1.0, NAN, 1.0, 2.0, INF, 1 - 2.0 ** -24, -0.0], device=dev), top_k=_ints([9] * 8, dev)).tolist()
    order = [sorted(r) for r in x.topk(9, 1).indices.tolist()]
    assert token == [order[i][0 if i in (0, 1, 2, 7) else -1] for i in range(8)]


@pytest.mark.parametrize("kind", ["f32", "f16"])
def test_sample_strides(dev, kind):
    x, u = _logits(6, 5001, kind, 8, dev)
    u = torch.tensor(u, device=dev)
    want = bq.bpdq_sample(x, u, top_p=torch.full((6,), 0.8, device=dev))
    for pad, at in ((8, 0), (1, 0), (7, 1)):
        wide = _inside(x, 5001 + pad, at)
        assert torch.equal(bq.bpdq_sample(wide, u, top_p=torch.full((6,), 0.8, device=dev)), want)
    big = torch.full((9,), -7, dtype=torch.int32, device=dev)
    bq.bpdq_sample(x, u, top_p=torch.full((6,), 0.8, device=dev), token=big[1:7])
    assert torch.equal(big[1:7], want) and big[0] == -7 and (big[7:] == -7).all()
    assert bq.bpdq_sample(x[:0], u[:0]).shape == (0,)


def test_sample_borders_everywhere(dev):
    """Values whose distances from the largest pass through every step of the histogram, kept up to any of them.  Weights are equal up to 2^-22 (distances
    are below 128, the temperature 10^9), so that top-p keeps the k that top_p = (k - 1/2) / n asks for, and the last kept has more than u leaves."""
    n, vocab = 1024, 8192
    x = torch.zeros(vocab, dtype=torch.float64)
    x[1:] = -torch.exp2(-5 + 12 * torch.arange(vocab - 1) / vocab)
    x = x.float().to(dev).repeat(n, 1)
    k = torch.arange(n, dtype=torch.int32) * 8 + torch.arange(n, dtype=torch.int32) % 8 + 1
    u, t = torch.full((n,), 1 - 2.0 ** -24, device=dev), torch.full((n,), 1e9, device=dev)
    assert torch.equal(bq.bpdq_sample(x, u, temperature=t, top_k=k.to(dev)).cpu(), k - 1)
    p = ((k.double() - 0.5) / vocab).float().to(dev)
    assert torch.equal(bq.bpdq_sample(x, u, temperature=t, top_p=p).cpu(), k - 1)


def test_sample_largest_vocabulary(dev):
    x = torch.zeros((2, 1 << 20), dtype=torch.float16, device=dev)
    x[1, -1] = 30.0
    _check_sample(x, [0.999, 0.5], dev=dev)
    _check_sample(x, [0.999, 0.5], p=[0.75, 0.75], dev=dev)
    _check_sample(x, [0.999, 0.5], k=[(1 << 20) - 1, 3], dev=dev)


# ------------------------------------------------------------------ streams and graphs

class Step:
    """What stands between the calls of a decoder layer, on buffers of its own."""

    def __init__(self, dev, n=5, d=256, f=192, vocab=9000):
        g = torch.Generator(device=dev).manual_seed(4)
        self.n, self.d = n, d
        self.x, self.r = (torch.randn((n, d), generator=g, device=dev).bfloat16() for _ in range(2))
        self.w = torch.ones(d, dtype=torch.bfloat16, device=dev)
        self.freq = torch.tensor(do.rotary_frequencies(64)[0], device=dev)
        self.pos, self.start = _ints(range(n), dev), _ints(range(n + 1), dev)
        p, c = _layer(2 * f, d, 2, 64, 1)
        self.gate = _on(p, c, dev)
        p, c = _layer(vocab, f, 3, 32, 2)
        self.head = _on(p, c, dev)
        self.u = torch.rand(n, generator=g, device=dev)
        self.k, self.p = _ints([0, 5, 40, 0, 2000][:n], dev), torch.tensor([0.9, 1.0, 0.5, 1.0, 0.97][:n], device=dev)

    def __call__(self):
        y, s = bq.bpdq_rms_norm(self.x, self.w, residual=self.r)
        codes, scales, _ = bq.bpdq_rms_norm_q8(self.x, self.w, residual=self.r, group=64)
        q, k = bq.bpdq_rotary(self.freq, self.pos, self.start, y.view(self.n, 4, 64), y.view(self.n, 4, 64)[:, :2], max_tok=1)
        z = bq.bpdq_gated_linear(*self.gate, 64, q.flatten(1))
        token, prob = bq.bpdq_sample(bq.bpdq_linear(*self.head, 32, z), self.u, top_k=self.k, top_p=self.p, want_prob=True)
        return s, codes, scales, k, z, token, prob

    def refresh(self, seed):
        g = torch.Generator(device=self.x.device).manual_seed(seed)
        self.x.copy_(torch.randn(self.x.shape, generator=g, device=self.x.device))
        self.u.copy_(torch.rand(self.n, generator=g, device=self.x.device))
        self.pos.add_(1)


def test_on_another_stream(dev):
    step = Step(dev)
    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_captured_and_replayed(dev):
    """Two captured graphs, replayed in turn on new inputs with eager calls between them, against the eager results."""
    step = Step(dev)
    step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        graphs.append((graph, out))
    for i in range(6):
        step.refresh(i)
        want = [t.clone() for t in step()]
        graph, out = graphs[i % 2]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i


# ------------------------------------------------------------------ all of them together

def test_the_example(dev):
    """The decoder of the example, prompts of two sequences and tokens behind them: the tokens are those that the served logits ask for.  Logits:
    every layer's attention is off by up to 4 % of its own size (the 8-bit cache: the attention's example), the other calls by roundings to
    bfloat16 (2^-9 of a value each, some ten to a layer), and what a layer adds to the residual stream is not larger than the stream: below
    4 % + 10 2^-9 = 6 % a layer, two layers, and the last norm and product 2 % more."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_decoder.py")
    spec = importlib.util.spec_from_file_location("serve_decoder", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    off, draws = example.main(["--tokens", "40", "--decode", "8", "--vocab", "500"])
    assert max(off) < 0.14
    for last, u, token in draws:
        host = _np(last)
        assert token[0] == int(np.argmax(host[0]))
        want, _, _, margin = do.sample(host[1], float(u[1]), float(np.float32(0.8)), 50, float(np.float32(0.95)))
        assert token[1] == want or margin <= 500 * 2.0 ** -43
