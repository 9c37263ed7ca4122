"""Performance cases of serving from the stored format: the product with bias, activation and residual, and the 8-bit cache.

A program that serves a quantized model runs, per layer and step, `bpdq_linear` for every weight matrix, `bpdq_kv_write` for the
keys and values of the new tokens and `bpdq_kv_attention` over the cache; `bpdq_kv_read` hands cached tokens to whoever wants
them in a floating type.  The listed cases are these calls at the layer shapes of `workloads.py` (28 query and 4 key heads of 128
make 3584 channels, 64 and 8 make 8192) and at the smallest of them; `draw` spreads sizes, head layouts, lengths and types.

The cache is in pages of `page` tokens; a page and key head hold `page * dim` codes and one scale.  A code is the value divided by
the scale, rounded, plus 128.  The scale is the largest magnitude of the first tokens written to the page, over 127, and doubles as
often as later tokens ask for it.  Within tiles of 64 tokens, token 16 g + 4 u + i, the codes of K lie as
[u][d / 64][d % 64 / 16][g][i][d % 16], those of V as [d / 16][g][d % 16][token % 16].
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
FLOOR = 2.0 ** -96                       # the least magnitude a page's scale is made for


def listed():
    return [
        # one token of 16 sequences into their pages, and those pages read back: launches are all of it
        {"name": "cache_step", "op": "cache", "n_seq": 16, "n_kv": 4, "dim": 128, "page": 64, "lo": 1, "hi": 1, "past": 1000,
         "all": False, "type": "bf16"},
        # the keys and values of a prompt
        {"name": "cache_prompt", "op": "cache", "n_seq": 1, "n_kv": 8, "dim": 128, "page": 64, "lo": 4096, "hi": 4096, "past": 0,
         "all": False, "type": "f16"},
        # ragged chunks that begin inside a page, read back with everything before them
        {"name": "cache_ragged", "op": "cache", "n_seq": 37, "n_kv": 5, "dim": 64, "page": 128, "lo": 1, "hi": 777, "past": 3000,
         "all": True, "type": "f32"},
        # one sequence, one token, a short cache: latency
        {"name": "attention_one", "op": "attention", "n_seq": 1, "n_q": 28, "n_kv": 4, "dim": 128, "page": 64, "lo": 1, "hi": 1,
         "kv_lo": 1000, "kv_hi": 1000, "window": 0, "type": "bf16"},
        # a batch of sequences of all lengths, one token each
        {"name": "attention_batch", "op": "attention", "n_seq": 32, "n_q": 64, "n_kv": 8, "dim": 128, "page": 64, "lo": 1, "hi": 1,
         "kv_lo": 1, "kv_hi": 16384, "window": 0, "type": "bf16"},
        # one long cache
        {"name": "attention_long", "op": "attention", "n_seq": 1, "n_q": 64, "n_kv": 8, "dim": 128, "page": 128, "lo": 1, "hi": 1,
         "kv_lo": 131071, "kv_hi": 131071, "window": 0, "type": "f16"},
        # a prompt against itself
        {"name": "attention_prompt", "op": "attention", "n_seq": 1, "n_q": 28, "n_kv": 4, "dim": 128, "page": 64, "lo": 4096,
         "hi": 4096, "kv_lo": 4096, "kv_hi": 4096, "window": 0, "type": "bf16"},
        # ragged chunks of prompts under a sliding window, heads of 64
        {"name": "attention_chunks", "op": "attention", "n_seq": 9, "n_q": 15, "n_kv": 5, "dim": 64, "page": 64, "lo": 3, "hi": 700,
         "kv_lo": 700, "kv_hi": 5000, "window": 1024, "type": "f16"},
        # one decoded token through a 7B attention layer with its bias
        {"name": "linear_token", "op": "linear", "n": 1, "d_out": 3584, "d_in": 3584, "bits": 2, "group": 128, "act": "none",
         "bias": True, "residual": False, "type": "bf16"},
        # a step of 16 sequences through the 7B up projection and its activation
        {"name": "linear_step", "op": "linear", "n": 16, "d_out": 18944, "d_in": 3584, "bits": 3, "group": 128, "act": "silu",
         "bias": False, "residual": False, "type": "f16"},
        # a chunk of odd length through the 72B attention output and its residual
        {"name": "linear_chunk", "op": "linear", "n": 333, "d_out": 8192, "d_in": 8192, "bits": 2, "group": 64, "act": "none",
         "bias": False, "residual": True, "type": "bf16"},
        # a prompt through the 7B up projection
        {"name": "linear_prompt", "op": "linear", "n": 4096, "d_out": 18944, "d_in": 3584, "bits": 2, "group": 128, "act": "gelu",
         "bias": True, "residual": False, "type": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["cache", "attention", "attention", "linear", "linear"])
    kind = rng.choice(["f16", "bf16"])
    if op == "linear":
        g = rng.choice([32, 64, 128, 256])
        d_in = g * _log_int(rng, 256 // g, 18944 // g)
        d_out = _log_int(rng, 64, min(18944, 6.7e7 / d_in))
        return {"op": op, "n": _log_int(rng, 1, 4096), "d_out": d_out, "d_in": d_in, "bits": rng.choice([1, 2, 2, 3, 4]), "group": g,
                "act": rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]), "bias": rng.random() < 0.5,
                "residual": rng.random() < 0.5, "type": kind}
    n_kv, dim, page = rng.choice([1, 2, 3, 4, 5, 8]), rng.choice([64, 128, 128, 256]), rng.choice([64, 128, 256])
    if op == "cache":
        n_seq = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, 8192 / n_seq)
        return {"op": op, "n_seq": n_seq, "n_kv": n_kv, "dim": dim, "page": page, "lo": rng.choice([1, hi]), "hi": hi,
                "past": rng.choice([0, _log_int(rng, 1, 32768 / n_seq)]), "all": rng.random() < 0.3, "type": rng.choice(["f32", "f16", "bf16"])}
    n_q = n_kv * rng.choice([1, 2, 3, 4, 7, 8])
    if rng.random() < 0.5:               # decoding, some with a few tokens a sequence
        n_seq = _log_int(rng, 1, 48)
        hi, kv_hi = rng.choice([1, 1, 1, 2, 5]), _log_int(rng, 64, 131072 / n_seq * min(1.0, 1024 / (n_kv * dim)))
    else:
        n_seq = _log_int(rng, 1, 8)
        kv_hi = _log_int(rng, 64, 4096 / math.sqrt(n_seq * max(1.0, n_q * dim / 3584)))
        hi = _log_int(rng, 16, kv_hi)
    return {"op": op, "n_seq": n_seq, "n_q": n_q, "n_kv": n_kv, "dim": dim, "page": page, "lo": rng.choice([1, hi]), "hi": hi,
            "kv_lo": rng.choice([hi, kv_hi]), "kv_hi": kv_hi, "window": rng.choice([0, 0, 0, _log_int(rng, 16, 2048)]), "type": kind}


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


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _normal(shape, g):
    return torch.randn(shape, generator=g, device="cuda")


def _stored_layer(case, g):
    """Planes and half-precision coefficients as the sweep leaves them: an offset and plane steps of about one, two, four and eight
    times the smallest."""
    d_out, d_in, k, n_grp = case["d_out"], case["d_in"], case["bits"], case["d_in"] // case["group"]
    planes = torch.randint(-(1 << 31), 1 << 31, (k, d_out, d_in // 32), generator=g, device="cuda", dtype=torch.int64)
    step = 0.08 / (1 << k) * (1.0 + 0.2 * _normal((k + 1, d_out, n_grp), g))
    mult = torch.tensor([-0.5 * ((1 << k) - 1)] + [float(1 << i) for i in range(k)], device="cuda")
    return planes.to(torch.int32), (step * mult[:, None, None]).half().contiguous()


def _cache(case, lengths, room, g):
    """A cache that holds lengths[b] tokens of sequence b, with pages in no order and room for room[b] tokens: keys with loud
    channels, values without, each page with the scale of its largest magnitude."""
    n_kv, dim, page = case["n_kv"], case["dim"], case["page"]
    need = [max(1, -(-r // page)) for r in room]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda")
    table = torch.zeros((len(room), max(need)), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    loud = torch.exp(0.5 * _normal((n_kv, 1, dim), g))
    out = {"table": table}
    for name, mult in (("k", loud), ("v", torch.ones_like(loud))):
        x = _normal((n_pages, n_kv, page, dim), g).mul_(mult)
        s = x.abs().amax((2, 3)) / 127.0
        code = (torch.round(x.div_(s[:, :, None, None])) + 128.0).to(torch.uint8)
        code = _lay_k(code) if name == "k" else _lay_v(code)
        out[name], out[name + "_scale"] = code.contiguous(), s
    return out


def prepare(case, seed):
    g = _gen(seed)
    kind = TYPES[case["type"]]
    if case["op"] == "linear":
        n, d_out, d_in = case["n"], case["d_out"], case["d_in"]
        planes, coefs = _stored_layer(case, g)
        s = {"case": case, "planes": planes, "coefs": coefs, "x": (_normal((n, d_in), g) * torch.exp(0.5 * _normal(d_in, g))).to(kind)}
        s["bias"] = _normal(d_out, g).to(kind) if case["bias"] else None
        s["residual"] = (4.0 * _normal((n, d_out), g)).to(kind) if case["residual"] else None
        return s
    n_seq, n_kv, dim, page = case["n_seq"], case["n_kv"], case["dim"], case["page"]
    if case["op"] == "cache":
        fresh = _lengths(n_seq, case["lo"], case["hi"])
        past = [max(0, case["past"] - 37 * b) for b in range(n_seq)]
        end = [p + f for p, f in zip(past, fresh)]
        s = {"case": case, **_cache(case, past, end, g)}
        first = [0 if case["all"] else p // page * page for p in past]
        x = _normal((sum(fresh), 2 * n_kv * dim), g).to(kind)          # keys and values of one product, side by side
        s["fresh_k"], s["fresh_v"] = x[:, :n_kv * dim].unflatten(1, (n_kv, dim)), x[:, n_kv * dim:].unflatten(1, (n_kv, dim))
        s["pos"], s["start"], s["most"] = _ints(past), _ints(_starts(fresh)), max(fresh)
        back = [e - f for e, f in zip(end, first)]
        s["back_pos"], s["back_start"], s["back_most"], s["back_sum"] = _ints(first), _ints(_starts(back)), max(back), sum(back)
        return s
    q_len = _lengths(n_seq, case["lo"], case["hi"])
    kv_len = [max(a, b) for a, b in zip(_lengths(n_seq, case["kv_lo"], case["kv_hi"]), q_len)]
    s = {"case": case, **_cache(case, kv_len, kv_len, g)}
    qkv = _normal((sum(q_len), (case["n_q"] + 2 * n_kv) * dim), g).to(kind)                # of one product, side by side
    s["q"] = qkv[:, :case["n_q"] * dim].unflatten(1, (case["n_q"], dim))
    s["kv_len"], s["start"], s["most"], s["kv_most"] = _ints(kv_len), _ints(_starts(q_len)), max(q_len), max(kv_len)
    return s


# ---------------------------------------------------------------------------- layout of the cache ---------

def _lay_k(code):
    """(..., page, dim) to the layout of K in a page."""
    *lead, page, dim = code.shape
    n = len(lead)
    x = code.reshape(*lead, page // 64, 4, 4, 4, dim // 64, 4, 16)                        # tile g u i c quarter byte
    return x.permute(*range(n), n, n + 2, n + 4, n + 5, n + 1, n + 3, n + 6).reshape(code.shape)


def _unlay_k(code):
    *lead, page, dim = code.shape
    n = len(lead)
    x = code.reshape(*lead, page // 64, 4, dim // 64, 4, 4, 4, 16)                        # tile u c quarter g i byte
    return x.permute(*range(n), n, n + 4, n + 1, n + 5, n + 2, n + 3, n + 6).reshape(code.shape)


def _lay_v(code):
    """(..., page, dim) to the layout of V in a page."""
    *lead, page, dim = code.shape
    n = len(lead)
    x = code.reshape(*lead, page // 64, 4, 16, dim // 16, 16)                             # tile g byte dt m
    return x.permute(*range(n), n, n + 3, n + 1, n + 4, n + 2).reshape(code.shape)


def _unlay_v(code):
    *lead, page, dim = code.shape
    n = len(lead)
    x = code.reshape(*lead, page // 64, dim // 16, 4, 16, 16)                             # tile dt g m byte
    return x.permute(*range(n), n, n + 2, n + 4, n + 1, n + 3).reshape(code.shape)


# ---------------------------------------------------------------------------- plain forms ---------

def _pow2(n):
    """2^n exactly, for whole numbers n."""
    return ((n.clamp(-126, 127) + 127) << 23).to(torch.int32).view(torch.float32)


def _act(v, act):
    if act == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v))
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _linear_plain(s):
    case = s["case"]
    k, d_out, nw = s["planes"].shape
    bit = torch.arange(32, device="cuda", dtype=torch.int32)
    b = ((s["planes"][..., None] >> bit) & 1).reshape(k, d_out, -1, case["group"])
    c = s["coefs"].float()[..., None]
    w = (c[0] + (c[1:] * b).sum(0)).reshape(d_out, 32 * nw)
    y = s["x"].float() @ w.t()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    y = _act(y, case["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def _pages(s, pos, end, most, page):
    """Of the pages that hold tokens pos[b] to end[b]: their sequences, their numbers there, and what the table says."""
    n = (most + page - 2) // page + 1
    first = pos // page
    at = first[:, None] + torch.arange(n, device="cuda")
    used = (at * page < end[:, None]) & (end > pos)[:, None]
    seq, t = torch.nonzero(used, as_tuple=True)
    at = at[seq, t]
    return seq, at, s["table"][seq, at].long()


def _write_plain(s, name, page, where):
    seq, at, phys = where
    x, start, pos = s["fresh_" + name], s["start"].long(), s["pos"].long()
    p = at[:, None] * page + torch.arange(page, device="cuda")                            # positions of the pages' slots
    end = pos + start[1:] - start[:-1]
    new = (p >= pos[seq][:, None]) & (p < end[seq][:, None])
    old = p < pos[seq][:, None]
    rows = torch.where(new, start[:-1][seq][:, None] + p - pos[seq][:, None], torch.zeros_like(p))
    v = torch.where(new[:, :, None, None], x[rows].float(), torch.zeros((), device="cuda")).transpose(1, 2)    # page head slot dim
    most = v.abs().amax((2, 3))
    had = old.any(1)[:, None]
    s0 = s[name + "_scale"][phys]
    m0, e0 = torch.frexp(127.0 * s0)
    m1, e1 = torch.frexp(most)
    up = torch.where(most > 127.0 * s0, (e1 - e0) + (m1 > m0).to(e1.dtype), torch.zeros_like(e1))
    scale = torch.where(had, s0 * _pow2(up), torch.clamp(most, min=FLOOR) * (1.0 / 127.0))
    fresh = torch.clamp(torch.round(v * (1.0 / scale)[:, :, None, None]), -127, 127)
    lay, unlay = (_lay_k, _unlay_k) if name == "k" else (_lay_v, _unlay_v)
    code = unlay(s[name][phys]).float() - 128.0
    code = torch.where(old[:, None, :, None], torch.round(code * _pow2(-up)[:, :, None, None]), code)
    code = torch.where(new[:, None, :, None], fresh, code)
    s[name][phys] = lay((code + 128.0).to(torch.uint8))
    s[name + "_scale"][phys] = scale


def _read_plain(s, name, page, where, kind):
    seq, at, phys = where
    start, pos = s["back_start"].long(), s["back_pos"].long()
    p = at[:, None] * page + torch.arange(page, device="cuda")
    row = start[:-1][seq][:, None] + p - pos[seq][:, None]
    keep = (p >= pos[seq][:, None]) & (row < start[1:][seq][:, None])
    code = (_unlay_k if name == "k" else _unlay_v)(s[name][phys]).float() - 128.0
    v = (code * s[name + "_scale"][phys][:, :, None, None]).transpose(1, 2)
    out = torch.empty((s["back_sum"],) + v.shape[2:], dtype=kind, device="cuda")
    out[row[keep]] = v[keep].to(kind)
    return out


def _cache_plain(s):
    page, kind = s["case"]["page"], s["fresh_k"].dtype
    start, pos = s["start"].long(), s["pos"].long()
    into = _pages(s, pos, pos + start[1:] - start[:-1], s["most"], page)
    _write_plain(s, "k", page, into)
    _write_plain(s, "v", page, into)
    start, pos = s["back_start"].long(), s["back_pos"].long()
    out_of = _pages(s, pos, pos + start[1:] - start[:-1], s["back_most"], page)
    return {"k": _read_plain(s, "k", page, out_of, kind), "v": _read_plain(s, "v", page, out_of, kind),
            "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _attention_plain(s):
    case, q = s["case"], s["q"]
    n_seq, n_q, n_kv, dim, page = case["n_seq"], case["n_q"], case["n_kv"], case["dim"], case["page"]
    n = -(-s["kv_most"] // page)
    phys = s["table"][:, :n].long()

    def dense(name, unlay):
        x = (unlay(s[name][phys]).float() - 128.0) * s[name + "_scale"][phys][..., None, None]
        return x.permute(0, 2, 1, 3, 4).reshape(n_seq, n_kv, n * page, dim)               # sequence head token dim

    start, kv_len = s["start"].long(), s["kv_len"].long()
    i = torch.arange(s["most"], device="cuda")
    q_len = start[1:] - start[:-1]
    there = i < q_len[:, None]
    rows = torch.where(there, start[:-1, None] + i, torch.zeros_like(there, dtype=torch.int64))
    x = q[rows].float().reshape(n_seq, s["most"], n_kv, n_q // n_kv, dim).permute(0, 2, 3, 1, 4)
    x = x.reshape(n_seq, n_kv, (n_q // n_kv) * s["most"], dim)
    z = (x * (1.0 / math.sqrt(dim))) @ dense("k", _unlay_k).transpose(2, 3).contiguous()
    at = (kv_len - q_len)[:, None] + i                                                    # the queries' positions
    t = torch.arange(n * page, device="cuda")
    seen = t <= at[:, :, None]
    if case["window"]:
        seen = seen & (t > at[:, :, None] - case["window"])
    z = z.reshape(n_seq, n_kv, n_q // n_kv, s["most"], n * page).masked_fill_(~seen[:, None, None], -math.inf)
    m = z.amax(4, keepdim=True)
    e = torch.exp(z.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)))
    total = e.sum(4, keepdim=True)
    o = e.reshape(n_seq, n_kv, -1, n * page) @ dense("v", _unlay_v)
    o = o.reshape(total.shape[:4] + (dim,)) / torch.where(total == 0, torch.ones_like(total), total)
    return o.permute(0, 3, 1, 2, 4).reshape(n_seq, s["most"], n_q, dim)[there].to(q.dtype)


# ---------------------------------------------------------------------------- one pass -------

def run(state):
    op, case = state["case"]["op"], state["case"]
    if not own:
        return {"linear": _linear_plain, "cache": _cache_plain, "attention": _attention_plain}[op](state)
    from paper_2602_04163_amd import binding as bq
    s = state
    if op == "linear":
        return bq.bpdq_linear(s["planes"], s["coefs"], case["group"], s["x"], bias=s["bias"], act=case["act"], residual=s["residual"])
    cache = bq.KvCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
    if op == "attention":
        return bq.bpdq_kv_attention(cache, s["table"], s["kv_len"], s["start"], s["q"], max_q=s["most"], max_kv=s["kv_most"],
                                    scale=1.0 / math.sqrt(case["dim"]), causal=True, window=case["window"])
    bq.bpdq_kv_write(cache, s["table"], s["pos"], s["start"], s["fresh_k"], s["fresh_v"], max_tok=s["most"])
    k, v = bq.bpdq_kv_read(cache, s["table"], s["back_pos"], s["back_start"], s["back_sum"], max_tok=s["back_most"],
                           dtype=s["fresh_k"].dtype)
    return {"k": k, "v": v, "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def work(case):
    size = 4.0 if case["type"] == "f32" else 2.0
    if case["op"] == "linear":
        n, d_out, d_in, k, g = case["n"], case["d_out"], case["d_in"], case["bits"], case["group"]
        return {"bytes": d_out * d_in * (k / 8.0 + 2.0 * (k + 1) / g) + size * n * (d_in + d_out * (2 if case["residual"] else 1)) +
                (size * d_out if case["bias"] else 0.0), "flops": 2.0 * n * d_out * d_in}
    n_seq, n_kv, dim, page = case["n_seq"], case["n_kv"], case["dim"], case["page"]
    if case["op"] == "cache":
        fresh = sum(_lengths(n_seq, case["lo"], case["hi"]))
        past = [max(0, case["past"] - 37 * b) for b in range(n_seq)]
        back = fresh + sum(p if case["all"] else p % page for p in past)
        # new values read and their codes written; codes read back and their values written
        return {"bytes": 2.0 * n_kv * dim * ((size + 1.0) * fresh + (size + 1.0) * back), "flops": 4.0 * n_kv * dim * (fresh + back)}
    q_len = _lengths(n_seq, case["lo"], case["hi"])
    kv_len = [max(a, b) for a, b in zip(_lengths(n_seq, case["kv_lo"], case["kv_hi"]), q_len)]
    w, pairs, tokens = case["window"], 0, 0
    for q, kv in zip(q_len, kv_len):
        full = w if w else kv + 1
        short = max(0, min(q, full - (kv - q) - 1))          # queries that see everything before them, the rest a full window
        pairs += short * (kv - q) + short * (short + 1) // 2 + (q - short) * full
        tokens += min(kv, q - 1 + w) if w else kv
    return {"bytes": 2.0 * size * case["n_q"] * dim * sum(q_len) + 2.0 * n_kv * (dim * tokens + 4.0 * tokens / page),
            "flops": 4.0 * dim * case["n_q"] * pairs}


# ---------------------------------------------------------------------------- 64 bits --------

def _linear64(case, s):
    k, g = case["bits"], case["group"]
    w = s["coefs"][0].double().repeat_interleave(g, 1)
    for i in range(k):
        word = s["planes"][i].repeat_interleave(32, 1)
        bits = torch.bitwise_right_shift(word, torch.arange(w.shape[1], device="cuda", dtype=torch.int32) % 32).remainder(2)
        w += s["coefs"][i + 1].double().repeat_interleave(g, 1) * bits
    y = s["x"].double() @ w.t().contiguous()
    if case["bias"]:
        y += s["bias"].double()
    if case["act"] == "relu":
        y = y.clamp(min=0)
    elif case["act"] == "gelu":
        y = y * torch.special.ndtr(y)
    elif case["act"] == "gelu_tanh":
        y = y * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3))
    elif case["act"] == "silu":
        y = y * torch.sigmoid(y)
    return y + s["residual"].double() if case["residual"] else y


def _at(page, dim, name):
    """Where the code of each slot and channel of a page lies."""
    t, d = torch.arange(page, device="cuda")[:, None], torch.arange(dim, device="cuda")[None, :]
    g, u, i = t % 64 // 16, t % 16 // 4, t % 4
    if name == "k":
        inside = (((u * (dim // 64) + d // 64) * 4 + d % 64 // 16) * 16 + 4 * g + i) * 16 + d % 16
    else:
        inside = ((d // 16 * 4 + g) * 16 + d % 16) * 16 + t % 16
    return t // 64 * 64 * dim + inside


def _codes64(s, name, phys, page, dim):
    """Codes of pages `phys` as (page of phys, head, slot, channel), in 64 bits."""
    flat = s[name][phys].flatten(2)
    return flat[:, :, _at(page, dim, name)].double() - 128.0


def _cache64(case, s):
    n_kv, dim, page = case["n_kv"], case["dim"], case["page"]
    pos, start, table = s["pos"].tolist(), s["start"].tolist(), s["table"].tolist()
    back, first = s["back_start"].tolist(), s["back_pos"].tolist()
    out = {}
    for name in ("k", "v"):
        fresh, scales, got = s["fresh_" + name].double(), s[name + "_scale"].double(), []
        for b in range(case["n_seq"]):
            end = pos[b] + start[b + 1] - start[b]
            n_page = -(-end // page)
            phys = torch.tensor(table[b][:n_page], device="cuda")
            code, sc = _codes64(s, name, phys, page, dim), s[name + "_scale"][phys].double()
            val = (code * sc[:, :, None, None]).transpose(1, 2).reshape(n_page * page, n_kv, dim)
            for j in range(pos[b] // page, n_page):
                lo, hi = max(pos[b], j * page), min(end, (j + 1) * page)
                x = fresh[start[b] + lo - pos[b]:start[b] + hi - pos[b]]
                most = x.abs().amax((0, 2))
                if lo > j * page:
                    ratio = most / (127.0 * sc[j])
                    grow = torch.where(ratio > 1, torch.exp2(torch.ceil(torch.log2(ratio))), torch.ones_like(ratio))
                    grow = torch.where(ratio > grow, 2 * grow, grow)
                    step = sc[j] * grow
                    val[j * page:lo] = torch.round((code[j] / grow[:, None, None])[:, :lo - j * page].transpose(0, 1)) * step[:, None]
                else:
                    step = most.clamp(min=FLOOR) / 127.0
                val[lo:hi] = torch.round(x / step[:, None]).clamp(-127, 127) * step[:, None]
                scales[phys[j]] = step
            got.append(val[first[b]:first[b] + back[b + 1] - back[b]])
        out[name], out[name + "_scale"] = torch.cat(got), scales
    return {n: out[n] for n in ("k", "v", "k_scale", "v_scale")}


def _attention64(case, s):
    n_q, n_kv, dim, page = case["n_q"], case["n_kv"], case["dim"], case["page"]
    start, kv_len = s["start"].tolist(), s["kv_len"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b in range(case["n_seq"]):
        n, kv = start[b + 1] - start[b], kv_len[b]
        phys = s["table"][b, :-(-kv // page)].long()
        for h in range(n_kv):
            k, v = [(_codes64({name: s[name][:, h:h + 1]}, name, phys, page, dim)[:, 0] *
                     s[name + "_scale"][phys, h].double()[:, None, None]).reshape(-1, dim)[:kv] for name in ("k", "v")]
            p = torch.arange(kv - n, kv, device="cuda")[:, None]
            t = torch.arange(kv, device="cuda")
            hidden = (t > p) | ((t <= p - case["window"]) if case["window"] else torch.zeros_like(t > p))
            for j in range(h * (n_q // n_kv), (h + 1) * (n_q // n_kv)):
                z = s["q"][start[b]:start[b + 1], j].double() @ k.t().contiguous() / math.sqrt(dim)
                out[start[b]:start[b + 1], j] = torch.softmax(z.masked_fill(hidden, -math.inf), 1) @ v
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _linear64, "cache": _cache64, "attention": _attention64}[case["op"]](case, s)
