"""Performance cases of what a served decoder layer has between its products and its attention, and of the step from logits to a token.

A program that serves a quantized model runs, per layer and step, `bpdq_rms_norm` on the sum of the residual stream and what the last
block adds, `bpdq_rotary` on the queries and keys of the new tokens before they go to the cache, and `bpdq_gated_linear` for the two
projections of its feed-forward block that share one input; at the end `bpdq_sample` picks the tokens.  The listed cases are these calls at
the layer shapes of `workloads.py` (28 query and 4 key heads of 128 make 3584 channels, 64 and 8 make 8192; a feed-forward block of 18944)
and a vocabulary of 152064; `draw` spreads sizes, layouts, types and masks.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
FLOOR = 2.0 ** -96                       # the least magnitude a scale of 8-bit codes is made for


def listed():
    return [
        # a step of 16 sequences between two blocks: launches are all of it
        {"name": "norm_step", "op": "norm", "n": 16, "d": 3584, "residual": "same", "codes": False, "group": 0, "offset": 0.0, "type": "bf16"},
        # a long prompt, the residual stream in 32 bits
        {"name": "norm_prompt", "op": "norm", "n": 4096, "d": 8192, "residual": "f32", "codes": False, "group": 0, "offset": 0.0, "type": "bf16"},
        # rows of a feed-forward block's width to 8 bits, as they are kept or sent, an odd number of them
        {"name": "norm_codes", "op": "norm", "n": 1023, "d": 18944, "residual": "none", "codes": True, "group": 128, "offset": 1.0,
         "type": "f16"},
        # one token of 16 sequences
        {"name": "rotary_step", "op": "rotary", "n_seq": 16, "n_q": 28, "n_kv": 4, "dim": 128, "rot": 128, "layout": "half", "lo": 1, "hi": 1,
         "past": 1000, "base": 1e6, "scaling": "none", "type": "bf16"},
        # a prompt that goes on behind a long past, with frequencies scaled for it
        {"name": "rotary_prompt", "op": "rotary", "n_seq": 1, "n_q": 64, "n_kv": 8, "dim": 128, "rot": 128, "layout": "half", "lo": 8192,
         "hi": 8192, "past": 120000, "base": 1e6, "scaling": "bands", "type": "f16"},
        # ragged chunks, neighbours as pairs, half of a head
        {"name": "rotary_ragged", "op": "rotary", "n_seq": 37, "n_q": 15, "n_kv": 5, "dim": 64, "rot": 32, "layout": "interleaved", "lo": 1,
         "hi": 777, "past": 3000, "base": 1e4, "scaling": "yarn", "type": "bf16"},
        # one decoded token through both projections of a feed-forward block
        {"name": "gated_token", "op": "gated", "n": 1, "f": 18944, "d_in": 3584, "bits": 2, "group": 128, "act": "silu", "bias": False,
         "type": "bf16"},
        # a chunk of odd length, finer groups, with biases
        {"name": "gated_chunk", "op": "gated", "n": 333, "f": 18944, "d_in": 3584, "bits": 3, "group": 64, "act": "gelu_tanh", "bias": True,
         "type": "f16"},
        # a prompt
        {"name": "gated_prompt", "op": "gated", "n": 4096, "f": 18944, "d_in": 3584, "bits": 2, "group": 128, "act": "silu", "bias": False,
         "type": "bf16"},
        # one sequence's next token: latency
        {"name": "sample_one", "op": "sample", "n": 1, "vocab": 152064, "filters": "both", "masked": 0.0, "type": "bf16"},
        # a batch whose requests differ in what they ask for
        {"name": "sample_batch", "op": "sample", "n": 64, "vocab": 152064, "filters": "mixed", "masked": 0.0, "type": "f32"},
        # many rows of a smaller, odd vocabulary under masks, no limit but probabilities
        {"name": "sample_masked", "op": "sample", "n": 256, "vocab": 32003, "filters": "p", "masked": 0.9, "type": "f16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["norm", "rotary", "gated", "sample"])
    if op == "norm":
        codes, d = rng.random() < 0.35, _log_int(rng, 64, 29568)
        group = rng.choice([0, 32, 64, 128, 256]) if codes else 0
        d = max(group, d // group * group) if group else d
        kind = rng.choice(["f16", "bf16"]) if codes else rng.choice(["f32", "f16", "bf16"])
        return {"op": op, "n": _log_int(rng, 1, min(8192, 3.3e7 / d)), "d": d, "residual": rng.choice(["none", "same", "f32"]),
                "codes": codes, "group": group, "offset": rng.choice([0.0, 0.0, 1.0]), "type": kind}
    if op == "rotary":
        dim, n_kv = rng.choice([64, 80, 128, 256]), rng.choice([1, 2, 3, 4, 5, 8])
        n_q = n_kv * rng.choice([1, 2, 3, 4, 7, 8])
        n_seq = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, 7.5e7 / (n_seq * (n_q + n_kv) * dim))
        return {"op": op, "n_seq": n_seq, "n_q": n_q, "n_kv": n_kv, "dim": dim, "rot": rng.choice([dim, dim, dim // 2, 2 * rng.randint(1, dim // 2)]),
                "layout": rng.choice(["half", "half", "interleaved"]), "lo": rng.choice([1, hi]), "hi": hi,
                "past": rng.choice([0, _log_int(rng, 1, 1 << 20)]), "base": rng.choice([1e4, 1e6]),
                "scaling": rng.choice(["none", "linear", "yarn", "bands"]), "type": rng.choice(["f32", "f16", "bf16"])}
    if op == "gated":
        g = rng.choice([32, 64, 128, 256])
        d_in = g * _log_int(rng, 256 // g, 8192 // g)
        f = _log_int(rng, 64, min(29568, 6.7e7 / d_in))
        return {"op": op, "n": _log_int(rng, 1, 4096), "f": f, "d_in": d_in, "bits": rng.choice([1, 2, 2, 3, 4]), "group": g,
                "act": rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu", "silu"]), "bias": rng.random() < 0.3,
                "type": rng.choice(["f16", "bf16"])}
    vocab = _log_int(rng, 1000, 262144)
    return {"op": op, "n": _log_int(rng, 1, min(512, 9.7e6 / vocab)), "vocab": vocab, "filters": rng.choice(["none", "k", "p", "both", "mixed"]),
            "masked": rng.choice([0.0, 0.0, 0.5, 0.99]), "type": rng.choice(["f32", "f16", "bf16"])}


# ---------------------------------------------------------------------------- inputs ---------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) % (1 << 62))
    return g


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _lengths(n, lo, hi):
    """n < 67 lengths over [lo, hi], both ends among them, out of order; they depend on the case alone."""
    return [lo + (hi - lo) * (67 * i % n) // (n - 1) for i in range(n)] if n > 1 else [hi]


def _normal(shape, g):
    return torch.randn(shape, generator=g, device="cuda")


def _frequencies(rot, base, scaling):
    """Radians per position of each pair in 64 bits, and the factor on cosine and sine: the base's powers, slowed down fourfold by `linear`; by
    `yarn` from one turn in 4096 positions down, not from 32 turns up, in steps between; by `bands` eightfold from one turn in 8192 down, not
    from four turns up."""
    i = np.arange(rot // 2, dtype=np.float64)
    f = base ** (-2.0 * i / rot)
    if scaling == "linear":
        return f / 4.0, 1.0
    if scaling == "yarn":
        at = [rot * math.log(4096 / (2 * math.pi * turns)) / (2 * math.log(base)) for turns in (32.0, 1.0)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
        slow = np.clip((i - lo) / (hi - lo if hi > lo else 0.001), 0.0, 1.0)
        return f / 4.0 * slow + f * (1.0 - slow), 0.1 * math.log(4.0) + 1.0
    if scaling == "bands":
        turns = 8192 * f / (2 * math.pi)
        fast = np.clip((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        return f / 8.0 * (1.0 - fast) + f * fast, 1.0
    return f, 1.0


def _filters(case, g):
    """What each row asks for: temperature, top_k, top_p, min_p (None: nobody asks), by its place in the batch."""
    n, kind = case["n"], case["filters"]
    row = torch.arange(n, device="cuda")
    t = 0.6 + 0.2 * (row % 5).float()
    k = (20 + 30 * (row % 4)).to(torch.int32)
    p = 0.85 + 0.03 * (row % 4).float()
    m = 0.02 + 0.01 * (row % 3).float()
    if kind == "none":
        return t, None, None, None
    if kind == "k":
        return t, k, None, None
    if kind == "p":
        return t, None, p, m
    if kind == "both":
        return t, k, p, None
    # greedy, temperature alone, top-k, top-p, both and min-p in turn
    ask = row % 6
    return (torch.where(ask == 0, torch.zeros_like(t), t), torch.where((ask == 2) | (ask == 4), k, torch.zeros_like(k)),
            torch.where((ask == 3) | (ask == 4), p, torch.ones_like(p)), torch.where(ask == 5, m, torch.zeros_like(m)))


def prepare(case, seed):
    g, kind = _gen(seed), TYPES[case["type"]]
    s = {"case": case}
    if case["op"] == "norm":
        n, d = case["n"], case["d"]
        loud = torch.exp(0.5 * _normal(d, g))
        s["x"] = (_normal((n, d), g) * loud).to(kind)
        wide = torch.float32 if case["residual"] == "f32" else kind
        s["residual"] = None if case["residual"] == "none" else (3.0 * _normal((n, d), g) * loud).to(wide)
        s["weight"] = (1.0 - case["offset"] + 0.3 * _normal(d, g)).to(kind)
    elif case["op"] == "rotary":
        fresh = _lengths(case["n_seq"], case["lo"], case["hi"])
        qkv = _normal((sum(fresh), (case["n_q"] + 2 * case["n_kv"]) * case["dim"]), g).to(kind)     # of one product, side by side
        at = case["n_q"] * case["dim"]
        s["q"] = qkv[:, :at].unflatten(1, (case["n_q"], case["dim"]))
        s["k"] = qkv[:, at:at + case["n_kv"] * case["dim"]].unflatten(1, (case["n_kv"], case["dim"]))
        s["pos"] = _ints([max(0, case["past"] - 37 * b) for b in range(case["n_seq"])])
        s["start"] = _ints([0] + list(np.cumsum(fresh)))
        s["most"] = max(fresh)
        freq, s["mscale"] = _frequencies(case["rot"], case["base"], case["scaling"])
        s["freq"] = torch.tensor(freq, dtype=torch.float64, device="cuda")
    elif case["op"] == "gated":
        n, f, d_in, k, n_grp = case["n"], case["f"], case["d_in"], case["bits"], case["d_in"] // case["group"]
        # planes and half-precision coefficients as the sweep leaves them for two layers stacked by rows: an offset and plane steps of about
        # one, two, four and eight times the smallest, so that the projections of the inputs below have a magnitude of about one
        planes = torch.randint(-(1 << 31), 1 << 31, (k, 2 * f, d_in // 32), generator=g, device="cuda", dtype=torch.int64)
        step = 3.0 / math.sqrt(d_in) / (1 << k) * (1.0 + 0.2 * _normal((k + 1, 2 * f, n_grp), g))
        mult = torch.tensor([-0.5 * ((1 << k) - 1)] + [float(1 << i) for i in range(k)], device="cuda")
        s["planes"], s["coefs"] = planes.to(torch.int32), (step * mult[:, None, None]).half().contiguous()
        s["x"] = (_normal((n, d_in), g) * torch.exp(0.5 * _normal(d_in, g))).to(kind)
        s["bias"] = (0.5 * _normal(2 * f, g)).to(kind) if case["bias"] else None
    else:
        n, v = case["n"], case["vocab"]
        x = 2.0 * _normal((n, v), g)
        likely = torch.randint(0, v, (n, 48), generator=g, device="cuda")
        x.scatter_add_(1, likely, 9.0 * torch.rand((n, 48), generator=g, device="cuda") + 2.0)
        if case["masked"]:               # what a grammar forbids
            masked = torch.rand((n, v), generator=g, device="cuda") < case["masked"]
            x.masked_fill_(masked.scatter_(1, likely[:, :1], False), -math.inf)
        s["logits"] = x.to(kind)
        s["u"] = torch.rand(n, generator=g, device="cuda")
        s["temperature"], s["top_k"], s["top_p"], s["min_p"] = _filters(case, g)
    return s


# ---------------------------------------------------------------------------- plain forms ---------

def _norm_plain(s):
    case, x = s["case"], s["x"]
    v = x.float() if s["residual"] is None else x.float() + s["residual"].float()
    y = v * (1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6)) * (case["offset"] + s["weight"].float())
    out = {}
    if s["residual"] is not None:
        out["sum"] = v.to(s["residual"].dtype)
    if not case["codes"]:
        out["y"] = y.to(x.dtype)
        return out
    y = y.unflatten(1, (-1, case["group"] or case["d"]))
    scale = torch.clamp(y.abs().amax(2), min=FLOOR) * (1.0 / 127.0)
    codes = torch.clamp(torch.round(y / scale[:, :, None]), -127, 127).to(torch.int8)
    out["y"] = (codes.float() * scale[:, :, None]).flatten(1).to(x.dtype)
    out["scale"] = scale
    return out


def _rotary_plain(s):
    case, kind = s["case"], s["q"].dtype
    start, rot = s["start"].long(), case["rot"]
    row = torch.arange(s["q"].shape[0], device="cuda")
    seq = (row[:, None] >= start[None, 1:]).sum(1)
    angle = (s["pos"].long()[seq] + row - start[seq]).double()[:, None] * s["freq"]
    c, n = (s["mscale"] * torch.cos(angle)).float()[:, None], (s["mscale"] * torch.sin(angle)).float()[:, None]

    def turned(x):
        part, rest = x[:, :, :rot].float(), x[:, :, rot:]
        if case["layout"] == "half":
            a, b = part[:, :, :rot // 2], part[:, :, rot // 2:]
            part = torch.cat((a * c - b * n, b * c + a * n), 2)
        else:
            a, b = part[:, :, 0::2], part[:, :, 1::2]
            part = torch.stack((a * c - b * n, b * c + a * n), 3).flatten(2)
        return torch.cat((part.to(kind), rest), 2)

    return {"q": turned(s["q"]), "k": turned(s["k"])}


def _act(v, act):
    if act == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v))
    if act == "gelu":
        return 0.5 * v * torch.erfc(v * -math.sqrt(0.5))
    if act == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _gated_plain(s):
    case = s["case"]
    k, rows, nw = s["planes"].shape
    bit = torch.arange(32, device="cuda", dtype=torch.int32)
    b = ((s["planes"][..., None] >> bit) & 1).reshape(k, rows, -1, case["group"])
    c = s["coefs"].float()[..., None]
    w = (c[0] + (c[1:] * b).sum(0)).reshape(rows, 32 * nw)
    y = s["x"].float() @ w.t()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return (_act(y[:, :case["f"]], case["act"]) * y[:, case["f"]:]).to(s["x"].dtype)


def _sample_plain(s):
    """In 64 bits: sums over a vocabulary decide whether a token is in, and which one is next."""
    x, n = s["logits"].double(), s["case"]["n"]
    t = s["temperature"].double()[:, None]
    most = x.amax(1, keepdim=True)
    w = torch.where(t > 0, torch.exp((x - most) / torch.where(t > 0, t, torch.ones_like(t))), (x == most).double())
    w, order = torch.sort(w, dim=1, descending=True, stable=True)
    place = torch.arange(w.shape[1], device="cuda")
    keep = w > 0
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        keep = keep & ((place < k) | (k <= 0))
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        cum = (w * keep).cumsum(1)
        keep = keep & ((cum - w < p * cum[:, -1:]) | (p >= 1))
    if s["min_p"] is not None:
        keep = keep & (w >= s["min_p"].double()[:, None])
    keep = keep & ((place < 1) | (t > 0))
    w = torch.zeros_like(w).scatter_(1, order, w * keep)
    cum = w.cumsum(1)
    token = (cum <= s["u"].double()[:, None] * cum[:, -1:]).sum(1, keepdim=True)
    return {"token": token[:, 0].to(torch.int32), "prob": (w.gather(1, token) / cum[:, -1:])[:, 0].float()}


# ---------------------------------------------------------------------------- one pass -------

def run(state):
    s, case = state, state["case"]
    op = case["op"]
    if not own:
        return {"norm": _norm_plain, "rotary": _rotary_plain, "gated": _gated_plain, "sample": _sample_plain}[op](s)
    from paper_2602_04163_amd import binding as bq
    if op == "rotary":
        q, k = bq.bpdq_rotary(s["freq"], s["pos"], s["start"], s["q"], s["k"], max_tok=s["most"], layout=case["layout"], mscale=s["mscale"])
        return {"q": q, "k": k}
    if op == "gated":
        return bq.bpdq_gated_linear(s["planes"], s["coefs"], case["group"], s["x"], bias=s["bias"], act=case["act"])
    if op == "sample":
        token, prob = bq.bpdq_sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                                     min_p=s["min_p"], want_prob=True)
        return {"token": token, "prob": prob}
    out = {}
    if case["codes"]:
        codes, scale, total = bq.bpdq_rms_norm_q8(s["x"], s["weight"], eps=1e-6, residual=s["residual"], offset=case["offset"],
                                                  group=case["group"])
        y = torch.empty_like(s["x"])
        torch.mul(codes.unflatten(1, scale.shape[1:] + (-1,)), scale[:, :, None], out=y.unflatten(1, scale.shape[1:] + (-1,)))
    else:
        y, total = bq.bpdq_rms_norm(s["x"], s["weight"], eps=1e-6, residual=s["residual"], offset=case["offset"])
    if total is not None:
        out["sum"] = total
    out["y"] = y
    if case["codes"]:
        out["scale"] = scale
    return out


def work(case):
    size = 4.0 if case["type"] == "f32" else 2.0
    if case["op"] == "norm":
        n, d = case["n"], case["d"]
        wide = {"none": 0.0, "same": size, "f32": 4.0}[case["residual"]]
        # the values of the codes, as they are returned, in place of the codes
        scales = 4.0 * n * d / (case["group"] or d) if case["codes"] else 0.0
        return {"bytes": n * d * (2.0 * size + 2.0 * wide) + size * d + scales, "flops": 6.0 * n * d}
    if case["op"] == "rotary":
        n, heads = sum(_lengths(case["n_seq"], case["lo"], case["hi"])), case["n_q"] + case["n_kv"]
        return {"bytes": 2.0 * size * n * heads * case["dim"], "flops": 3.0 * n * heads * case["rot"]}
    if case["op"] == "gated":
        n, f, d_in, k, g = case["n"], case["f"], case["d_in"], case["bits"], case["group"]
        return {"bytes": 2.0 * f * d_in * (k / 8.0 + 2.0 * (k + 1) / g) + size * n * (d_in + f) + (2.0 * size * f if case["bias"] else 0.0),
                "flops": 4.0 * n * f * d_in}
    return {"bytes": case["n"] * (size * case["vocab"] + 28.0), "flops": 10.0 * case["n"] * case["vocab"]}


# ---------------------------------------------------------------------------- 64 bits --------

def _norm64(case, s):
    v = s["x"].double()
    if s["residual"] is not None:
        v = v + s["residual"].double()
    out = {} if s["residual"] is None else {"sum": v}
    y = v / torch.linalg.vector_norm(v, dim=1, keepdim=True).square().div(case["d"]).add(1e-6).sqrt()
    y = y * (s["weight"].double() + case["offset"])
    if case["codes"]:
        block = y.reshape(case["n"], -1, case["group"] or case["d"])
        step = block.abs().max(2, keepdim=True).values.clamp(min=FLOOR) / 127
        y = (step * torch.round(block / step)).reshape(y.shape)
        return {**out, "y": y, "scale": step[:, :, 0]}
    return {**out, "y": y}


def _rotary64(case, s):
    start, pos, half = s["start"].tolist(), s["pos"].tolist(), case["rot"] // 2
    where = torch.cat([torch.arange(p, p + b - a, device="cuda") for p, a, b in zip(pos, start, start[1:])]).double()
    turn = torch.polar(torch.full((len(where), half), s["mscale"], dtype=torch.float64, device="cuda"), torch.outer(where, s["freq"]))
    i = torch.arange(half, device="cuda")
    first, second = (i, i + half) if case["layout"] == "half" else (2 * i, 2 * i + 1)
    out = {}
    for name in ("q", "k"):
        y = s[name].double()
        z = torch.complex(y[:, :, first], y[:, :, second]) * turn[:, None]
        y[:, :, first], y[:, :, second] = z.real, z.imag
        out[name] = y
    return out


def _gated64(case, s):
    f, g = case["f"], case["group"]
    both = []
    for at in (0, f):
        w = s["coefs"][0, at:at + f].double().repeat_interleave(g, 1)
        for i in range(case["bits"]):
            word = s["planes"][i, at:at + f].repeat_interleave(32, 1)
            bits = torch.bitwise_right_shift(word, torch.arange(w.shape[1], device="cuda", dtype=torch.int32) % 32).remainder(2)
            w += s["coefs"][i + 1, at:at + f].double().repeat_interleave(g, 1) * bits
        y = s["x"].double() @ w.t().contiguous()
        both.append(y + s["bias"][at:at + f].double() if case["bias"] else y)
    y, act = both[0], case["act"]
    if act == "relu":
        y = y.clamp(min=0)
    elif act == "gelu":
        y = y * torch.special.ndtr(y)
    elif act == "gelu_tanh":
        y = y * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3))
    elif act == "silu":
        y = y * torch.sigmoid(y)
    return y * both[1]


def _sample64(case, s):
    x, u = s["logits"].double().cpu().numpy(), s["u"].double().cpu().numpy()
    ask = [None if s[name] is None else s[name].double().cpu().numpy() for name in ("temperature", "top_k", "top_p", "min_p")]
    token, prob = np.zeros(case["n"], dtype=np.int32), np.zeros(case["n"])
    for r in range(case["n"]):
        t, k, p, m = [None if a is None else a[r] for a in ask]
        if not t > 0:
            token[r], prob[r] = int(np.argmax(x[r])), 1.0
            continue
        live = np.flatnonzero(x[r] > -np.inf)
        live = live[np.argsort(-x[r][live], kind="stable")]
        if k is not None and k > 0:
            live = live[:int(k)]
        w = np.exp((x[r][live] - x[r][live[0]]) / t)
        n = len(live)
        if p is not None and p < 1:
            n = min(n, 1 + int(np.searchsorted(np.cumsum(w), p * w.sum(), side="left")))
        if m is not None:
            n = min(n, int((w >= m).sum()))
        by = np.argsort(live[:n])
        cum = np.cumsum(w[:n][by])
        at = int(np.searchsorted(cum, u[r] * cum[-1], side="right"))
        token[r], prob[r] = live[:n][by][at], w[:n][by][at] / cum[-1]
    return {"token": torch.tensor(token, device="cuda"), "prob": torch.tensor(prob, device="cuda")}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _norm64, "rotary": _rotary64, "gated": _gated64, "sample": _sample64}[case["op"]](case, s)
