"""Plain numpy oracle of the serving operators: the product with bias, activation and residual, the 8-bit key/value cache
(codes and scales in fp32, step for step, as include/bpdq.h defines them) and attention over it (fp64)."""
from __future__ import annotations

import math

import numpy as np

FLOOR = np.float32(2.0 ** -96)
_INV127 = np.float32(1.0) / np.float32(127.0)


# ------------------------------------------------------------------ layout of a page and head
def k_place(page: int, dim: int) -> np.ndarray:
    """(page, dim) array: byte offset of the code of slot t, channel d in K."""
    t, d = np.arange(page)[:, None], np.arange(dim)[None, :]
    tile, g, u, i = t // 64, t % 64 // 16, t % 16 // 4, t % 4
    return tile * 64 * dim + (((u * (dim // 64) + d // 64) * 4 + d % 64 // 16) * 16 + 4 * g + i) * 16 + d % 16


def v_place(page: int, dim: int) -> np.ndarray:
    t, d = np.arange(page)[:, None], np.arange(dim)[None, :]
    return t // 64 * 64 * dim + ((d // 16 * 4 + t % 64 // 16) * 16 + d % 16) * 16 + t % 16


class Cache:
    """One of K and V: codes (n_pages, n_kv, page, dim) by slot and channel, scales (n_pages, n_kv)."""

    def __init__(self, n_pages, n_kv, page, dim):
        self.code = np.full((n_pages, n_kv, page, dim), 128, np.uint8)
        self.scale = np.zeros((n_pages, n_kv), np.float32)
        self.page = page

    def write(self, table, pos, x):
        """Tokens x (n, n_kv, dim) of one sequence at position pos."""
        x = np.asarray(x, np.float32)
        n, at = len(x), 0
        while at < n:
            slot = (pos + at) % self.page
            take = min(self.page - slot, n - at)
            p = table[(pos + at) // self.page]
            for h in range(x.shape[1]):
                self._write(p, h, slot, x[at:at + take, h])
            at += take

    def _write(self, p, h, slot, x):
        with np.errstate(all="ignore"):
            amax = np.abs(x).max()
            s0 = self.scale[p, h]
            if not np.isfinite(x).all():
                self.scale[p, h] = np.nan
                return
            if slot == 0:
                s = np.float32(max(amax, FLOOR) * _INV127)
            else:
                s, j = s0, 0
                while amax > np.ldexp(np.float32(127.0) * s0, j):
                    j += 1
                if j:
                    s = np.ldexp(s0, j)
                    old = self.code[p, h, :slot].astype(np.float64) - 128.0
                    self.code[p, h, :slot] = (np.rint(old * 2.0 ** -j) + 128).astype(np.uint8)
            self.scale[p, h] = s
            if np.isfinite(s):
                q = np.rint(x * (np.float32(1.0) / s))
                self.code[p, h, slot:slot + len(x)] = (np.clip(q, -127, 127) + 128).astype(np.uint8)

    def dense(self, table, n):
        """The first n tokens of a sequence, (n, n_kv, dim) in fp64."""
        pages = [int(p) for p in table[: -(-n // self.page)]]
        v = (self.code[pages].astype(np.float64) - 128.0) * self.scale[pages].astype(np.float64)[:, :, None, None]
        return v.transpose(0, 2, 1, 3).reshape(-1, v.shape[1], v.shape[3])[:n]


# ------------------------------------------------------------------ the product
def dequant(planes, coefs, group):
    """What in fp64 from planes (k, d_out, nw) uint32 and coefficients (k + 1, d_out, d_in / group)."""
    k, d_out, nw = planes.shape
    bits = ((planes[..., None] >> np.arange(32, dtype=np.uint32)) & 1).reshape(k, d_out, 32 * nw)
    c = np.repeat(coefs.astype(np.float64), group, axis=2)
    w = c[0].copy()
    for i in range(k):
        w += c[i + 1] * bits[i]
    return w


def act(v, name):
    with np.errstate(over="ignore"):
        if name == "relu":
            return np.maximum(v, 0.0)
        if name == "gelu":
            return 0.5 * v * (1.0 + np.vectorize(math.erf)(v / math.sqrt(2.0)))
        if name == "gelu_tanh":
            return 0.5 * v * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
        if name == "silu":
            return v / (1.0 + np.exp(-v))
    return v


def linear(planes, coefs, group, x, bias=None, name="none", residual=None):
    """Returns the result and sum |What| |x| + |bias|, which rounding errors are measured by."""
    w, x = dequant(planes, coefs, group), x.astype(np.float64)
    y, size = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        y, size = y + bias.astype(np.float64), size + np.abs(bias.astype(np.float64))
    y = act(y, name)
    return (y if residual is None else y + residual.astype(np.float64)), size


# ------------------------------------------------------------------ attention
def attention(q, k, v, scale, causal=True, window=0):
    """q (n, n_q, dim), k, v (kv, n_kv, dim) of one sequence, the last query at position kv - 1.  Returns out, lse, sum p |v| and the
    largest |scale| sum |q| |k| of each row, all in fp64."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    n, n_q, dim = q.shape
    kv, n_kv = k.shape[:2]
    out, size = np.zeros((n, n_q, dim)), np.zeros((n, n_q, dim))
    lse, reach = np.full((n, n_q), -np.inf), np.zeros((n, n_q))
    p_at, t_at = np.arange(kv - n, kv)[:, None], np.arange(kv)[None, :]
    seen = np.ones((n, kv), bool)
    if causal:
        seen &= t_at <= p_at
    if window:
        seen &= t_at > p_at - window
    for h in range(n_q):
        g = h // (n_q // n_kv)
        for i in range(n):
            t = np.flatnonzero(seen[i])
            if not len(t):
                continue
            z = scale * (k[t, g] @ q[i, h])
            reach[i, h] = abs(scale) * (np.abs(k[t, g]) @ np.abs(q[i, h])).max()
            m = z.max()
            e = np.exp(z - m)
            out[i, h], size[i, h] = e @ v[t, g] / e.sum(), e @ np.abs(v[t, g]) / e.sum()
            lse[i, h] = m + math.log(e.sum())
    return out, lse, size, reach
