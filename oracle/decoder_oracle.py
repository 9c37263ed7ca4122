"""Plain numpy oracle, in fp64, of what a served decoder layer has around its products and its attention: the norm, rotary positions, the gated
product, and the choice of the next token.  Definitions: include/bpdq.h."""
from __future__ import annotations

import math

import numpy as np

from oracle import serving_oracle as so

FLOOR = 2.0 ** -96


def rms_norm(x, residual=None, weight=None, offset=0.0, eps=1e-6):
    """The sum and the norm."""
    s = x.astype(np.float64) if residual is None else x.astype(np.float64) + residual.astype(np.float64)
    with np.errstate(invalid="ignore"):
        y = s / np.sqrt((s * s).mean(1, keepdims=True) + eps)
    w = np.ones(x.shape[1]) if weight is None else weight.astype(np.float64)
    return s, y * (offset + w)


def scales(y, group=0):
    n, d = y.shape
    return np.maximum(np.abs(y).reshape(n, -1, group or d).max(2), FLOOR) / 127.0


def rotary_frequencies(rot, base=10000.0, scaling="plain", factor=1.0, low=1.0, high=32.0, original=4096):
    """Radians per position, one pair at a time."""
    if scaling == "ntk":
        base = base * factor ** (rot / (rot - 2))
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        turns = original * f / (2 * math.pi)
        if scaling == "linear":
            f = f / factor
        elif scaling == "bands":
            # all of it where it turns `high` times, a factor less at `low`, in proportion between
            share = min(1.0, max(0.0, (turns - low) / (high - low)))
            f = share * f + (1 - share) * f / factor
        elif scaling == "yarn":
            def pair(n):                 # where base^(-2 i / rot) original / 2 pi = n
                return rot / 2 * math.log(original / (2 * math.pi * n), base)
            first, last = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), rot - 1)
            share = 1 - min(1.0, max(0.0, (i - first) / (last - first if last > first else 0.001)))
            f = share * f + (1 - share) * f / factor
        out.append(f)
    return np.array(out), 0.1 * math.log(factor) + 1.0 if scaling == "yarn" else 1.0


def rotary(x, position, freq, layout="half", mscale=1.0, inverse=False):
    """x (n, heads, dim) with row i at position[i]."""
    y = x.astype(np.float64)
    half = len(freq)
    for i in range(half):
        a, b = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
        t = position * float(freq[i]) * (-1 if inverse else 1)
        c, s = mscale * np.cos(t)[:, None], mscale * np.sin(t)[:, None]
        y[:, :, a], y[:, :, b] = x[:, :, a] * c - x[:, :, b] * s, x[:, :, b] * c + x[:, :, a] * s
    return y


def gated(planes, coefs, group, x, bias=None, name="silu"):
    """Returns the result, gate and up before activation and product, and the sizes |W| |x| + |bias| of both and the roots of their sums of
    squares, which rounding errors are measured by."""
    f = planes.shape[1] // 2
    parts, sizes, roots = [], [], []
    for at in (0, f):
        p, c = planes[:, at:at + f], coefs[:, at:at + f]
        y, size = so.linear(p, c, group, x, None if bias is None else bias[at:at + f])
        parts.append(y)
        sizes.append(size)
        roots.append(np.sqrt((x.astype(np.float64) ** 2) @ (so.dequant(p, c, group) ** 2).T))
    return so.act(parts[0], name) * parts[1], parts, sizes, roots


def sample(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row.  Returns token, prob, the kept indices, and how far from a border the choice was: the least distance of a running sum from what it
    was compared with, the largest weight being 1."""
    x = x.astype(np.float64)
    live = [i for i in range(len(x)) if x[i] > -np.inf]
    if not live:
        return -1, 0.0, [], 1.0
    live.sort(key=lambda i: -x[i])       # stable: ties by index
    if not temperature > 0:
        return live[0], 1.0, live[:1], 1.0
    top = x[live[0]]
    w = {i: 1.0 if x[i] == top else 0.0 if top == np.inf else math.exp((x[i] - top) / temperature) for i in live}
    if top_k > 0:
        live = live[:top_k]
    margin = 1.0
    if top_p < 1:
        total, run, n = math.fsum(w[i] for i in live), 0.0, 0
        while n == 0 or (run < top_p * total and n < len(live)):
            run += w[live[n]]
            n += 1
            margin = min(margin, abs(run - top_p * total))
        live = live[:n]
    if min_p > 0:
        margin = min([margin] + [abs(w[i] - min_p) for i in live if w[i] < 1])
        live = [i for i in live if w[i] >= min(min_p, 1.0)]
    kept = sorted(live)
    total, run = math.fsum(w[i] for i in kept), 0.0
    u = min(max(u, 0.0), 1.0)
    token = [i for i in kept if w[i] > 0][-1]
    for i in kept:
        before, run = run, run + w[i]
        if before > 0:
            margin = min(margin, abs(before - u * total))
        if run > u * total and w[i] > 0:
            token = i
            margin = min(margin, abs(run - u * total)) if i != kept[-1] else margin
            break
    return token, w[token] / total, kept, margin
