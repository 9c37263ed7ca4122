"""An attention block served from what the pass stored: its four projections quantized with `bpdq_quantize_layer`, then a prompt and decoded
tokens through `bpdq_linear`, `bpdq_kv_write`, `bpdq_kv_attention` and `bpdq_linear` with the residual, with keys and values in 8 bits.

    python examples/serve_attention.py [--tokens 300] [--decode 40] [--heads 8] [--kv-heads 2] [--dim 64]

Weights and activations are synthetic (`workloads.py`).  Both the attention's output and the block's are compared with the same block on the
dequantized weights in 64 bits with an exact cache.  They are compared apart because the residual is some 25 times the size of what the block
adds here: in the sum, the residual's rounding to bfloat16 would hide what the cache and the attention do.  (Positions enter Q and K between
the projection and the cache in a real model; that is the model's part and is left out.)
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_04163_amd import binding as bq  # noqa: E402
from paper_2602_04163_amd import workloads as wk  # noqa: E402


def quantize(d_out, d_in, index, dev):
    """One projection through the pass: planes, half-precision coefficients, group."""
    wl = wk.WORKLOADS["cfg2_qwen7b_attn"].scaled(index=10 + index, d_out=d_out, d_in=d_in, n_tok=2048, chunk=2048, group=64, bits=4)
    X = wk.make_activation_chunk(wl, 0, wk.channel_scales(wl, dev), dev)
    H = torch.zeros((d_in, d_in), device=dev)
    bq.bpdq_hessian_accumulate(X, H)
    U, dead, info = bq.bpdq_prepare(H, wl.damp)
    out = bq.bpdq_quantize_layer(wk.make_weight(wl, dev), U, dead,
                                 bq.make_params(wl.bits, wl.group, wl.block, wl.refine_iters, wl.alpha, coef_fp16=True))
    assert int(info) == 0
    return out["planes"], bq.bpdq_coefs_to_fp16(out["coefs"]), wl.group


class Attention:
    """The served block, for any mix of prompts and single tokens."""

    def __init__(self, qkv, o, heads, kv_heads, dim, n_seq, most, page=64):
        self.qkv, self.o, self.heads, self.kv_heads, self.dim = qkv, o, heads, kv_heads, dim
        dev, per = qkv[0].device, -(-most // page)
        self.cache = bq.KvCache.empty(n_seq * per, kv_heads, dim, page, dev)
        self.table = torch.randperm(n_seq * per, device=dev).to(torch.int32).view(n_seq, per)
        self.len = [0] * n_seq

    def __call__(self, x, counts):
        """x: counts[0] tokens of sequence 0, counts[1] of sequence 1, ...; returns the attention's output and x + its projection."""
        dev = x.device
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
        start = [sum(counts[:b]) for b in range(len(counts) + 1)]
        pos, self.len = self.len, [a + n for a, n in zip(self.len, counts)]
        split = (self.heads * self.dim, self.kv_heads * self.dim, self.kv_heads * self.dim)
        q, k, v = bq.bpdq_linear(*self.qkv, x).split(split, 1)
        k, v = k.unflatten(1, (self.kv_heads, self.dim)), v.unflatten(1, (self.kv_heads, self.dim))
        bq.bpdq_kv_write(self.cache, self.table, ints(pos), ints(start), k, v, max(counts))
        out = bq.bpdq_kv_attention(self.cache, self.table, ints(self.len), ints(start), q.unflatten(1, (self.heads, self.dim)),
                                   max(counts), max(self.len))
        out = out.flatten(1)
        return out, bq.bpdq_linear(*self.o, out, residual=x)


def exact(x, qkv, o, heads, kv_heads, dim):
    """The block on one whole sequence in 64 bits, with the dequantized weights."""
    w = [bq.bpdq_dequant_fp16(*layer).double() for layer in (qkv, o)]
    x = x.double()
    q, k, v = (x @ w[0].t()).split((heads * dim, kv_heads * dim, kv_heads * dim), 1)
    n, out = len(x), []
    hidden = torch.ones((n, n), dtype=torch.bool, device=x.device).triu(1)
    for h in range(heads):
        g = h // (heads // kv_heads)
        z = q[:, h * dim:(h + 1) * dim] @ k[:, g * dim:(g + 1) * dim].t().contiguous() * dim ** -0.5
        out.append(torch.softmax(z.masked_fill(hidden, float("-inf")), 1) @ v[:, g * dim:(g + 1) * dim])
    out = torch.cat(out, 1)
    return out, x + out @ w[1].t()


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=300, help="prompt of the first sequence; the second has half of it")
    ap.add_argument("--decode", type=int, default=40, help="tokens decoded one by one behind the prompts")
    ap.add_argument("--heads", type=int, default=8)
    ap.add_argument("--kv-heads", type=int, default=2)
    ap.add_argument("--dim", type=int, default=64)
    a = ap.parse_args(argv)
    dev = torch.device("cuda:0")
    d = a.heads * a.dim
    qkv = quantize((a.heads + 2 * a.kv_heads) * a.dim, d, 0, dev)
    o = quantize(d, d, 1, dev)
    prompts = [a.tokens, max(1, a.tokens // 2)]
    block = Attention(qkv, o, a.heads, a.kv_heads, a.dim, len(prompts), a.tokens + a.decode)
    g = torch.Generator(device=dev).manual_seed(1)
    x = [torch.randn((n + a.decode, d), generator=g, device=dev).bfloat16() for n in prompts]
    served = [r.split(prompts) for r in block(torch.cat([t[:n] for t, n in zip(x, prompts)]), prompts)]
    got = [[[whole[b]] for whole in served] for b in range(len(prompts))]
    for i in range(a.decode):
        for r, rows in enumerate(block(torch.stack([t[n + i] for t, n in zip(x, prompts)]), [1] * len(prompts))):
            for b in range(len(prompts)):
                got[b][r].append(rows[b:b + 1])
    errors = []
    for t, parts in zip(x, got):
        out, y = exact(t, qkv, o, a.heads, a.kv_heads, a.dim)
        off = [float((torch.cat(p).double() - w).norm() / w.norm()) for p, w in zip(parts, (out, y))]
        share = float((y - t.double()).norm() / y.norm())
        print(f"{len(t)} tokens: from 64 bits, attention {off[0]:.2e}, block {off[1]:.2e} of its norm (the block adds {share:.2e} of it)")
        errors.append((off[0], off[1], share))
    return errors


if __name__ == "__main__":
    main()
