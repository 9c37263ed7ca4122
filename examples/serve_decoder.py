"""A decoder served from what the pass stored, tokens in and tokens out: every layer is `bpdq_rms_norm`, `bpdq_linear` (Q, K and V in one), `bpdq_rotary`,
`bpdq_kv_write`, `bpdq_kv_attention`, `bpdq_linear`, `bpdq_rms_norm` on the sum with the residual, `bpdq_gated_linear` (gate and up quantized in one sweep
by `bpdq_quantize_layers`) and `bpdq_linear`; behind the last one a norm, the product with the vocabulary and `bpdq_sample`.

    python examples/serve_decoder.py [--layers 2] [--tokens 60] [--decode 12] [--vocab 1000]

Weights are synthetic (`workloads.py`) and quantized on synthetic activations, so what it says means nothing; the logits are compared with
the same decoder on the dequantized weights in 64 bits with an exact cache, and the tokens are those that the served logits ask for.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_04163_amd import binding as bq  # noqa: E402
from paper_2602_04163_amd import workloads as wk  # noqa: E402

EPS = 1e-6


def quantize(sizes, d_in, index, dev):
    """Layers that share one input, through the pass in one sweep: planes, half-precision coefficients, group."""
    wl = wk.WORKLOADS["cfg2_qwen7b_attn"].scaled(index=20 + index, d_out=sum(sizes), d_in=d_in, n_tok=2048, chunk=2048, group=64, bits=4)
    X = wk.make_activation_chunk(wl, 0, wk.channel_scales(wl, dev), dev)
    H = torch.zeros((d_in, d_in), device=dev)
    bq.bpdq_hessian_accumulate(X, H)
    U, dead, info = bq.bpdq_prepare(H, wl.damp)
    ends = [sum(sizes[:i + 1]) for i in range(len(sizes))]
    W = wk.make_weight(wl, dev)
    W *= d_in ** -0.5 / W.std()
    out = bq.bpdq_quantize_layers(W, ends, U, dead, bq.make_params(wl.bits, wl.group, wl.block, wl.refine_iters, wl.alpha, coef_fp16=True))
    assert int(info) == 0
    return out["planes"], bq.bpdq_coefs_to_fp16(out["coefs"]), wl.group


class Decoder:
    """The served model; a step takes any mix of prompts and single tokens."""

    def __init__(self, layers, heads, kv_heads, dim, ff, vocab, n_seq, most, dev, page=64):
        d = heads * dim
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        g = torch.Generator(device=dev).manual_seed(3)
        self.embed = torch.randn((vocab, d), generator=g, device=dev).bfloat16()
        weight = lambda: (1 + 0.1 * torch.randn(d, generator=g, device=dev)).bfloat16()  # noqa: E731
        self.layers = []
        for n in range(layers):
            self.layers.append({"norm1": weight(), "qkv": quantize([heads * dim, kv_heads * dim, kv_heads * dim], d, 4 * n, dev),
                                "o": quantize([d], d, 4 * n + 1, dev), "norm2": weight(), "gate_up": quantize([ff, ff], d, 4 * n + 2, dev),
                                "down": quantize([d], ff, 4 * n + 3, dev), "cache": bq.KvCache.empty(n_seq * -(-most // page), kv_heads, dim, page, dev)})
        self.norm, self.head = weight(), quantize([vocab], d, 4 * layers, dev)
        freq, self.mscale = bq.bpdq_rotary_frequencies(dim, 1e4, "yarn", factor=4.0, original=64)
        self.freq = freq.to(dev)
        self.table = torch.randperm(n_seq * -(-most // page), device=dev).to(torch.int32).view(n_seq, -1)
        self.len = [0] * n_seq

    def __call__(self, tokens, counts):
        """tokens: counts[0] of sequence 0, counts[1] of sequence 1, ...; returns their logits."""
        dev = tokens.device
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
        start, pos = ints([sum(counts[:b]) for b in range(len(counts) + 1)]), ints(self.len)
        self.len = [a + n for a, n in zip(self.len, counts)]
        end, most = ints(self.len), max(counts)
        split = (self.heads * self.dim, self.kv_heads * self.dim, self.kv_heads * self.dim)
        x, h = self.embed[tokens], None                   # what the last block adds, and the residual stream
        for layer in self.layers:
            y, h = bq.bpdq_rms_norm(x, layer["norm1"], EPS, residual=h) if h is not None else (bq.bpdq_rms_norm(x, layer["norm1"], EPS)[0], x)
            q, k, v = (t.unflatten(1, (-1, self.dim)) for t in bq.bpdq_linear(*layer["qkv"], y).split(split, 1))
            bq.bpdq_rotary(self.freq, pos, start, q, k, most, mscale=self.mscale, Q_out=q, K_out=k)
            bq.bpdq_kv_write(layer["cache"], self.table, pos, start, k, v, most)
            out = bq.bpdq_kv_attention(layer["cache"], self.table, end, start, q, most, max(self.len))
            y, h = bq.bpdq_rms_norm(bq.bpdq_linear(*layer["o"], out.flatten(1)), layer["norm2"], EPS, residual=h, S=h if h is not x else None)
            x = bq.bpdq_linear(*layer["down"], bq.bpdq_gated_linear(*layer["gate_up"], y, act="silu"))
        return bq.bpdq_linear(*self.head, bq.bpdq_rms_norm(x, self.norm, EPS, residual=h)[0])

    def exact(self, tokens):
        """Logits of one whole sequence in 64 bits, with the dequantized weights."""
        w = lambda layer: bq.bpdq_dequant_fp16(*layer).double().t().contiguous()  # noqa: E731
        norm = lambda x, g: x / (x.square().mean(1, keepdim=True) + EPS).sqrt() * g.double()  # noqa: E731
        h, n, dim = self.embed[tokens].double(), len(tokens), self.dim
        angle = torch.polar(torch.full((), self.mscale, dtype=torch.float64, device=h.device),
                            torch.outer(torch.arange(n, device=h.device).double(), self.freq))
        hidden = torch.ones((n, n), dtype=torch.bool, device=h.device).triu(1)

        def turned(x):
            z = torch.complex(x[:, :dim // 2], x[:, dim // 2:]) * angle
            return torch.cat((z.real, z.imag), 1)

        for layer in self.layers:
            qkv = (norm(h, layer["norm1"]) @ w(layer["qkv"])).split(dim, 1)
            q, k, v = qkv[:self.heads], qkv[self.heads:-self.kv_heads], qkv[-self.kv_heads:]
            out = []
            for i in range(self.heads):
                j = i // (self.heads // self.kv_heads)
                z = turned(q[i]) @ turned(k[j]).t().contiguous() * dim ** -0.5
                out.append(torch.softmax(z.masked_fill(hidden, float("-inf")), 1) @ v[j])
            h = h + torch.cat(out, 1) @ w(layer["o"])
            gate, up = (norm(h, layer["norm2"]) @ w(layer["gate_up"])).chunk(2, 1)
            h = h + (gate * torch.sigmoid(gate) * up) @ w(layer["down"])
        return norm(h, self.norm) @ w(self.head)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--tokens", type=int, default=60, help="prompt of the first sequence; the second has half of it")
    ap.add_argument("--decode", type=int, default=12, help="tokens sampled one by one behind the prompts")
    ap.add_argument("--vocab", type=int, default=1000)
    a = ap.parse_args(argv)
    dev = torch.device("cuda:0")
    prompts = [a.tokens, max(1, a.tokens // 2)]
    model = Decoder(a.layers, 8, 2, 64, 768, a.vocab, len(prompts), a.tokens + a.decode, dev)
    g = torch.Generator(device=dev).manual_seed(5)
    tokens = [torch.randint(0, a.vocab, (n,), generator=g, device=dev) for n in prompts]
    ask = {"temperature": torch.tensor([0.0, 0.8], device=dev), "top_k": torch.tensor([0, 50], dtype=torch.int32, device=dev),
           "top_p": torch.tensor([1.0, 0.95], device=dev)}       # the first sequence greedily
    logits = model(torch.cat(tokens), prompts)
    served = [[logits[n - 1:n]] for n in (prompts[0], sum(prompts))]
    draws = []
    for i in range(a.decode):
        last = torch.cat([s[-1] for s in served])
        u = torch.rand(len(prompts), generator=g, device=dev)
        token = bq.bpdq_sample(last, u, **ask)
        draws.append((last, u, token))
        tokens = [torch.cat((t, token[b:b + 1].long())) for b, t in enumerate(tokens)]
        logits = model(token.long(), [1] * len(prompts))
        for b in range(len(prompts)):
            served[b].append(logits[b:b + 1])
    off = []
    for t, s, n in zip(tokens, served, prompts):
        want = model.exact(t)[n - 1:]
        off.append(float((torch.cat(s).double() - want).norm() / want.norm()))
        print(f"{n} tokens and {a.decode} more: logits {off[-1]:.2e} of their norm from 64 bits; {t[n:].tolist()}")
    return off, draws


if __name__ == "__main__":
    main()
