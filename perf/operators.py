"""Timed operators of the serving side: what answering with a quantised model calls.

``listed()`` names twelve cases over the whole range; ``draw()`` gives more of the same ranges.
Kinds (``kind``):

  linear     a served layer on any number of tokens, bias, activation and residual in its epilogue
             (``kronq_online_linear``)
  grouped    the served layers of a mixture of experts on rows sorted by expert
             (``kronq_online_grouped``)
  append     new keys and values into a cache held in 4 bits (``kronq_cache_append``)
  attention  attention over that cache, of single tokens and of whole prompts
             (``kronq_cache_attention``)

With ``own`` false the same operators run as elementary torch operations in fp32 (the grid of the
cache in 64 bits).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
MIN_SCALE = 2.0 ** -100  # the smallest scale of a cache row


def listed():
    lin = {"kind": "linear", "group": 128, "rot_in": True, "rot_out": True, "bias": False,
           "act": "none", "residual": False, "x": "bf16", "y": "bf16"}
    moe = {**lin, "kind": "grouped"}
    att = {"kind": "attention", "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "rotate": True}
    app = {"kind": "append", "kv_heads": 8, "dim": 128, "page": 64, "rotate": True, "x": "bf16"}
    return [
        # one token through the attention output of an 8B block, added to the hidden state
        {"name": "linear_one_token", **lin, "d_out": 4096, "d_in": 4096, "bits": 4, "rows": 1,
         "residual": True},
        # a decode batch through the gate of the same block, 3 bits (as allocated), odd batch
        {"name": "linear_batch_gate", **lin, "d_out": 14336, "d_in": 4096, "bits": 3, "rows": 23,
         "act": "silu"},
        # a prompt through the down projection at 2 bits: 28 * 512 inputs, an odd length
        {"name": "linear_prompt_down", **lin, "d_out": 4096, "d_in": 14336, "bits": 2,
         "rows": 1337, "residual": True},
        # prompts of a batch through q_proj
        {"name": "linear_prompts_q", **lin, "d_out": 4096, "d_in": 4096, "bits": 4, "rows": 8192},
        # an unrotated 8-bit layer of odd output size in full precision (a scoring head)
        {"name": "linear_head_fp32", **lin, "d_out": 1001, "d_in": 4096, "bits": 8, "rows": 300,
         "rot_out": False, "bias": True, "x": "fp32", "y": "fp32"},
        # a decode batch routed to two of eight experts each
        {"name": "grouped_decode", **moe, "d_out": 14336, "d_in": 4096, "bits": 4, "experts": 8,
         "rows": 32, "act": "silu", "ragged": 1},
        # a prompt routed over many small experts, back into the hidden state
        {"name": "grouped_prompt", **moe, "d_out": 2048, "d_in": 1024, "bits": 4, "experts": 64,
         "rows": 8000, "ragged": 2},
        # the new tokens of a decode batch, one of each sequence
        {"name": "append_decode", **app, "tokens": 64, "ragged": 3},
        # the keys and values of a batch of prompts
        {"name": "append_prompts", **app, "tokens": 16000, "ragged": 4},
        # one new token of one sequence
        {"name": "attention_one", **att, "seqs": 1, "context": 1111, "queries": 1, "ragged": 5},
        # a decode batch over long contexts of different lengths, 70B heads
        {"name": "attention_decode", **att, "heads": 64, "seqs": 48, "context": 16384,
         "queries": 1, "ragged": 6},
        # prompts of different lengths packed one after another
        {"name": "attention_prompts", **att, "seqs": 6, "context": 2048, "queries": 2048,
         "ragged": 7},
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, even over its logarithm."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(("linear", "linear", "grouped", "append", "attention", "attention"))
    ragged = rng.randrange(1 << 30)
    if kind in ("linear", "grouped"):
        rot_in, rot_out = rng.random() < 0.8, rng.random() < 0.8
        lim = 14336 if kind == "linear" else 4096
        turned = [d for d in (256, 448, 512, 896, 1024, 1792, 2048, 3584, 4096, 7168, 8192, 14336)
                  if d <= lim]
        d_in = (rng.choice([d for d in turned if d % 128 == 0]) if rot_in
                else 128 * _spread(rng, 1, lim // 128))
        d_out = rng.choice(turned) if rot_out else _spread(rng, 33, lim)
        most_rows = min(8192, (1 << (37 if kind == "linear" else 35)) // (d_in * d_out))
        c = {"kind": kind, "d_out": d_out, "d_in": d_in, "bits": rng.choice((2, 3, 4, 8)),
             "group": rng.choice((128, 128, d_in)), "rot_in": rot_in, "rot_out": rot_out,
             "bias": rng.random() < 0.4, "act": rng.choice(("none", "none", "relu", "gelu", "silu")),
             "residual": rng.random() < 0.4, "x": rng.choice(("bf16", "bf16", "fp32")),
             "y": rng.choice(("bf16", "bf16", "fp32")), "rows": _spread(rng, 1, most_rows)}
        if kind == "grouped":
            c["experts"] = _spread(rng, 2, 64)
            c["ragged"] = ragged
        return c
    if kind == "append":
        return {"kind": kind, "kv_heads": rng.choice((1, 2, 4, 8)), "dim": rng.choice((64, 128)),
                "page": rng.choice((16, 32, 64, 128)), "rotate": rng.random() < 0.7,
                "x": rng.choice(("bf16", "bf16", "fp32")), "tokens": _spread(rng, 1, 16000),
                "ragged": ragged}
    kv = rng.choice((1, 2, 4, 8))
    queries = rng.choice((1, 1, _spread(rng, 2, 2048)))
    context = max(queries, _spread(rng, 1, 2048 if queries > 16 else 16384))
    return {"kind": kind, "kv_heads": kv,
            "heads": kv * rng.choice([n for n in (1, 3, 4, 7, 8) if queries <= 16 or kv * n <= 32]),
            "dim": rng.choice((64, 128)), "page": rng.choice((16, 32, 64, 128)),
            "rotate": rng.random() < 0.7, "queries": queries, "context": context,
            "seqs": _spread(rng, 1, 6 if queries > 16 else 48), "ragged": ragged}


# ---- sizes that follow from a case ---------------------------------------------------------------
def _counts(c):
    """Rows of each expert: a skewed router, some experts without any, a few rows of padding."""
    r = random.Random(c["ragged"])
    weight = [0.0 if r.random() < 0.1 else math.exp(0.6 * r.gauss(0, 1)) for _ in range(c["experts"])]
    weight[0] = max(weight[0], 0.5)
    rows = c["rows"] - (c["rows"] // 16 if r.random() < 0.5 else 0)
    total, left, out = sum(weight), rows, []
    for w in weight:
        n = min(left, round(rows * w / total))
        out.append(n)
        left -= n
    out[0] += left
    return out


def _lengths(c):
    """(tokens in the cache, new tokens) of each sequence."""
    r = random.Random(c["ragged"])
    out = []
    for i in range(c["seqs"]):
        length = c["context"] if i == 0 else max(1, round(c["context"] * r.uniform(0.1, 1.0)))
        new = c["queries"] if i == 0 else max(1, round(c["queries"] * r.uniform(0.2, 1.0)))
        out.append((length, min(new, length)))
    return out


def work(c):
    if c["kind"] in ("linear", "grouped"):
        size = {"bf16": 2, "fp32": 4}
        counts = _counts(c) if c["kind"] == "grouped" else [c["rows"]]
        rows, used = sum(counts), sum(n > 0 for n in counts)
        layer = c["d_out"] * c["d_in"] * c["bits"] / 8 + 8 * c["d_out"] * (c["d_in"] // c["group"])
        layer += 4 * (c["d_in"] + c["d_out"] * (2 if c["bias"] else 1))
        per_row = c["d_in"] * size[c["x"]] + c["d_out"] * size[c["y"]] * (2 if c["residual"] else 1)
        return {"bytes": used * layer + rows * per_row, "flops": 2 * rows * c["d_in"] * c["d_out"]}
    row = c["kv_heads"] * 2 * (c["dim"] / 2 + 4)  # a token's codes, scales and zeros
    if c["kind"] == "append":
        values = c["tokens"] * c["kv_heads"] * c["dim"] * 2
        return {"bytes": values * ({"bf16": 2, "fp32": 4}[c["x"]] + 4) + c["tokens"] * (row + 8),
                "flops": values * 8}
    seqs = _lengths(c)
    seen = sum(n * (length - n) + n * (n + 1) // 2 for length, n in seqs)
    return {"bytes": sum(length for length, _ in seqs) * row
            + 2 * 2 * sum(n for _, n in seqs) * c["heads"] * c["dim"],
            "flops": 4 * seen * c["heads"] * c["dim"]}


# ---- inputs ---------------------------------------------------------------------------------------
def _dtype(name):
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def _factor28(d):
    return d % 28 == 0 and (d // 28) & (d // 28 - 1) == 0


def _pack(codes, bits):
    """Runs of 32 codes as little-endian strings of `bits` words."""
    q = codes.unflatten(-1, (-1, 32)).to(torch.int64)
    words = []
    for k in range(bits):
        word = torch.zeros_like(q[..., 0])
        for j in range(32):
            at = j * bits - 32 * k
            if -bits < at < 32:
                word |= (q[..., j] << at if at >= 0 else q[..., j] >> -at) & 0xFFFFFFFF
        words.append(word)
    w = torch.stack(words, -1).flatten(-2)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def _prepare_linear(c, g):
    experts = c.get("experts", 1)
    d_out, d_in, bits = c["d_out"], c["d_in"], c["bits"]
    top = 2 ** bits - 1
    ng = d_in // c["group"]

    def normal(*size):
        return torch.randn(*size, generator=g, device=DEV)

    # codes of min-max grids of normal values, group by group
    packed = torch.stack([_pack((normal(d_out, d_in) * (top / 5.4) + top / 2).round_().clamp_(0, top)
                                .to(torch.uint8), bits) for _ in range(experts)]).flatten(0, 1)
    s = {"case": c, "packed": packed,
         "scales": torch.exp(0.2 * normal(experts * d_out, ng)) * (0.108 / top),
         "zeros": (normal(experts * d_out, ng) * 0.3 + top / 2).round_().clamp_(0, top)}

    # multipliers sign / s of both sides; the 28-point factors are orthogonal
    def mul(d):
        return torch.exp(0.5 * normal(experts, d)) * torch.where(normal(experts, d) < 0, -1.0, 1.0)

    s["mul_in"], s["mul_out"] = mul(d_in), mul(d_out)
    for side, d in (("in", d_in), ("out", d_out)):
        turn = c["rot_" + side] and _factor28(d)
        s["q28_" + side] = torch.linalg.qr(normal(experts, 28, 28))[0].contiguous() if turn else None
    # activations with a few strong channels
    strong = torch.where(torch.rand(d_in, generator=g, device=DEV) < 0.005, 20.0, 1.0)
    s["x"] = (normal(c["rows"], d_in) * strong).to(_dtype(c["x"]))
    s["bias"] = normal(experts, d_out) if c["bias"] else None
    s["residual"] = normal(c["rows"], d_out).to(_dtype(c["y"])) if c["residual"] else None
    if c["kind"] == "grouped":
        ends = np.cumsum([0] + _counts(c))
        s["offsets"] = torch.tensor(ends, dtype=torch.int32, device=DEV)
        s["most"] = int(max(np.diff(ends)))
        s["y"] = torch.zeros(c["rows"], d_out, dtype=_dtype(c["y"]), device=DEV)
    else:
        for name in ("mul_in", "mul_out", "q28_in", "q28_out", "bias"):
            s[name] = s[name][0] if s[name] is not None else None
    return s


def _cache(c, g, pages):
    """Codes, and scales with zeros, as the cache holds them (bell-shaped codes)."""
    kv, dim, page = c["kv_heads"], c["dim"], c["page"]
    words = pages * kv * 2 * page * dim // 8
    codes = torch.zeros(words, dtype=torch.int32, device=DEV)
    for j in range(8):
        v = torch.randn(words, generator=g, device=DEV, dtype=torch.float16)
        codes |= (v * 2.7 + 7.5).round_().clamp_(0, 15).to(torch.int32) << (4 * j)
    rows = pages * kv * 2 * page
    scale = (torch.exp(0.2 * torch.randn(rows, generator=g, device=DEV)) * 0.37).to(torch.bfloat16)
    zero = (torch.randn(rows, generator=g, device=DEV) * 0.8 + 7.5).round_().clamp_(0, 15)
    params = (scale.view(torch.int16).to(torch.int32) << 16) | zero.to(torch.int32)
    return codes.view(pages, kv, 2, page * dim // 8), params.view(pages, kv, 2, page)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    if case["kind"] in ("linear", "grouped"):
        return _prepare_linear(case, g)
    kv, dim, page = case["kv_heads"], case["dim"], case["page"]
    r = random.Random(seed)
    s = {"case": case}
    if case["kind"] == "append":
        tokens = case["tokens"]
        pages = -(-tokens // page) + 2
        s["codes"], s["params"] = _cache(case, g, pages)
        # whole and broken pages in any order
        order = torch.randperm(pages * page // 4, generator=g, device=DEV)
        slots = (order[:, None] * 4 + torch.arange(4, device=DEV)).flatten()[:tokens]
        s["slots"] = slots.to(torch.int64).contiguous()
        strong = torch.where(torch.rand(kv, dim, generator=g, device=DEV) < 0.03, 8.0, 1.0)
        for name in ("k", "v"):
            v = torch.randn(tokens, kv, dim, generator=g, device=DEV) * strong
            s[name] = v.to(_dtype(case["x"]))
            s[name + "_hat"] = torch.empty(tokens, kv, dim, device=DEV)
        return s
    seqs = _lengths(case)
    need = [-(-length // page) for length, _ in seqs]
    pages = sum(need) + 3
    s["codes"], s["params"] = _cache(case, g, pages)
    order = list(range(pages))
    r.shuffle(order)
    table = [[order.pop() for _ in range(n)] + [0] * (max(need) - n) for n in need]
    s["table"] = torch.tensor(table, dtype=torch.int32, device=DEV)
    s["lengths"] = torch.tensor([n for n, _ in seqs], dtype=torch.int32, device=DEV)
    s["starts"] = torch.tensor(np.cumsum([0] + [n for _, n in seqs]), dtype=torch.int32, device=DEV)
    s["most"] = max(n for _, n in seqs)
    s["q"] = torch.randn(sum(n for _, n in seqs), case["heads"], dim, generator=g,
                         device=DEV).to(torch.bfloat16)
    return s


# ---- plain forms ----------------------------------------------------------------------------------
def _hadamard(n, dtype=torch.float32):
    h = torch.ones(1, 1, dtype=dtype, device=DEV)
    while h.shape[0] < n:
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)))
    return h


def _turn(x, q28):
    """(Q28 (x) H_m) / sqrt(m), or H_d / sqrt(d), on the last axis of x [..., rows, d]."""
    d = x.shape[-1]
    m = d if q28 is None else d // 28
    a = 1 << (m.bit_length() // 2)
    if q28 is not None:
        x = q28.unsqueeze(-3) @ x.unflatten(-1, (28, m))
    h = x.reshape(*x.shape[:-1], -1, a, m // a) if q28 is not None else x.unflatten(-1, (a, m // a))
    h = _hadamard(a) @ h @ _hadamard(m // a)
    return h.reshape(*x.shape[:-2], d) * m ** -0.5 if q28 is not None else h.flatten(-2) * m ** -0.5


def _unpack(packed, bits):
    """Codes of packed strings, as fp32."""
    w = packed.unflatten(-1, (-1, bits))
    j = torch.arange(32, device=DEV) * bits
    at, off = j // 32, (j % 32).to(torch.int32)
    below = torch.clamp(32 - off, max=bits)  # bits of a code in its first word
    low = (w[..., at] >> off) & ((1 << below) - 1)
    high = (w[..., torch.clamp(at + 1, max=bits - 1)] & ((1 << (bits - below)) - 1)) << below
    return (low | high).flatten(-2).to(torch.float32)


def _act(z, name):
    if name == "relu":
        return torch.clamp(z, min=0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _plain_linear(s):
    c = s["case"]
    lead = (c["experts"],) if c["kind"] == "grouped" else ()
    q = _unpack(s["packed"], c["bits"]).unflatten(-1, (-1, c["group"]))
    w = ((q - s["zeros"][..., None]) * s["scales"][..., None]).flatten(-2)
    w = w.reshape(*lead, c["d_out"], c["d_in"])
    x = s["x"].float()
    if lead:  # each expert's rows, as many as the fullest expert has
        offsets = s["offsets"].to(torch.int64)
        at = offsets[:-1, None] + torch.arange(s["most"], device=DEV)
        x = x[torch.clamp(at, max=c["rows"] - 1)]
    x = x * s["mul_in"].unsqueeze(-2)
    if c["rot_in"]:
        x = _turn(x, s["q28_in"])
    y = x @ w.transpose(-1, -2)
    if c["rot_out"]:
        q28 = s["q28_out"]
        y = _turn(y, q28.transpose(-1, -2) if q28 is not None else None)
    y = y * s["mul_out"].unsqueeze(-2)
    if s["bias"] is not None:
        y = y + s["bias"].unsqueeze(-2)
    y = _act(y, c["act"])
    if lead:  # back to the order of the rows; rows of no expert keep what they hold
        row = torch.arange(c["rows"], device=DEV)
        e = torch.searchsorted(offsets, row, right=True) - 1
        in_range = e < c["experts"]
        e = torch.clamp(e, max=c["experts"] - 1)
        y = y[e, torch.clamp(row - offsets[e], max=s["most"] - 1)]
    if s["residual"] is not None:
        y = y + s["residual"].float()
    y = y.to(_dtype(c["y"]))
    return torch.where(in_range[:, None], y, s["y"]) if lead else y


def _grid(v, rotate):
    """Codes, scale and zero of the rows of v, and the values they stand for. In 64 bits: a value
    next to a border between two codes goes to one of them."""
    r = v.double()
    if rotate:
        r = r @ _hadamard(r.shape[-1], torch.float64) * r.shape[-1] ** -0.5
    low, high = torch.clamp(r.amin(-1), max=0), torch.clamp(r.amax(-1), min=0)
    scale = torch.clamp((high - low) / 15, min=MIN_SCALE)
    drop = (1 << 45) - 1  # of the 52 bits of a double's fraction, bf16 keeps 7: rounded up
    scale = ((scale.view(torch.int64) + drop) & ~drop).view(torch.float64)
    zero = torch.clamp(torch.round(-low / scale), max=15)
    codes = torch.clamp(torch.round(r / scale[..., None]) + zero[..., None], 0, 15)
    hat = (scale[..., None] * (codes - zero[..., None])).to(torch.float32)
    nibbles = codes.to(torch.int32).unflatten(-1, (-1, 8)) << (4 * torch.arange(8, device=DEV))
    params = scale.to(torch.float32).view(torch.int32) | zero.to(torch.int32)
    return nibbles.sum(-1).to(torch.int32), params, hat


def _plain_append(s):
    c = s["case"]
    page = c["page"]
    at, off = s["slots"] // page, s["slots"] % page
    kc, kp, k_hat = _grid(s["k"], c["rotate"])
    vc, vp, v_hat = _grid(s["v"], c["rotate"])
    pages = s["codes"].shape[0]
    kc_all = s["codes"][:, :, 0].view(pages, c["kv_heads"], page, -1)
    vc_all = s["codes"][:, :, 1].view(pages, c["kv_heads"], page // 4, -1, 4)
    kc_all[at, :, off] = kc
    vc_all[at, :, off // 4, :, off % 4] = vc
    s["params"][:, :, 0][at, :, off] = kp
    s["params"][:, :, 1][at, :, off] = vp
    return {"k": k_hat, "v": v_hat, "codes": s["codes"], "params": s["params"]}


def _read_cache(s, part):
    """Keys (part 0) or values (part 1) of every sequence, fp32 [seqs, kv_heads, tokens, dim]."""
    c = s["case"]
    table = s["table"].to(torch.int64)
    words = s["codes"][:, :, part][table]  # [seqs, pages, kv_heads, words of a page]
    words = (words.unflatten(-1, (c["page"] // 4, -1, 4)).transpose(-1, -2) if part
             else words.unflatten(-1, (c["page"], -1)))
    words = words.flatten(3, -2).transpose(1, 2).flatten(2, 3)
    nibbles = (words[..., None] >> (4 * torch.arange(8, device=DEV, dtype=torch.int32))) & 15
    params = s["params"][:, :, part][table].transpose(1, 2).flatten(2, 3)
    scale = (params & -65536).view(torch.float32)
    zero = (params & 0xFFFF).to(torch.float32)
    return (nibbles.flatten(-2).to(torch.float32) - zero[..., None]) * scale[..., None]


def _plain_attention(s):
    c = s["case"]
    heads, kv, dim = c["heads"], c["kv_heads"], c["dim"]
    k, v = _read_cache(s, 0), _read_cache(s, 1)
    starts, lengths = s["starts"].to(torch.int64), s["lengths"].to(torch.int64)
    # queries [seqs, kv_heads, heads of one kv head, most, dim], padded
    step = torch.arange(s["most"], device=DEV)
    at = starts[:-1, None] + step
    q = s["q"].float()
    if c["rotate"]:
        q = q @ _hadamard(dim) * dim ** -0.5
    q = q[torch.clamp(at, max=q.shape[0] - 1)].unflatten(2, (kv, -1)).permute(0, 2, 3, 1, 4)
    scores = q.flatten(2, 3) @ k.transpose(-1, -2) * dim ** -0.5
    scores = scores.unflatten(2, (heads // kv, -1))
    new = starts[1:] - starts[:-1]
    last = (lengths - new)[:, None] + step  # the last token a query sees
    hidden = torch.arange(k.shape[2], device=DEV) > last[..., None]
    scores.masked_fill_(hidden[:, None, None], -math.inf)
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    p /= p.sum(-1, keepdim=True)
    o = (p.flatten(2, 3) @ v).unflatten(2, (heads // kv, -1))
    o = o.permute(0, 3, 1, 2, 4).flatten(2, 3)  # [seqs, most, heads, dim]
    row = torch.arange(s["q"].shape[0], device=DEV)
    b = torch.searchsorted(starts, row, right=True) - 1
    o = o[b, row - starts[b]]
    if c["rotate"]:
        o = o @ _hadamard(dim) * dim ** -0.5
    return o.to(torch.bfloat16)


# ---- the framework's calls ------------------------------------------------------------------------
def _flags(c):
    from paper_2607_07964_amd import kronq as K
    return (K.ROT_IN if c["rot_in"] else 0) | (K.ROT_OUT if c["rot_out"] else 0)


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"linear": _plain_linear, "grouped": _plain_linear, "append": _plain_append,
                "attention": _plain_attention}[c["kind"]](s)
    from paper_2607_07964_amd import kronq as K
    if c["kind"] == "linear":
        return K.kronq_online_linear(
            s["packed"], s["scales"], s["zeros"], c["bits"], c["group"], c["d_in"], s["mul_in"],
            s["mul_out"], s["q28_in"], s["q28_out"], s["x"], bias=s["bias"], act=c["act"],
            residual=s["residual"], out_dtype=_dtype(c["y"]), flags=_flags(c))
    if c["kind"] == "grouped":
        return K.kronq_online_grouped(
            s["packed"], s["scales"], s["zeros"], c["bits"], c["group"], c["d_in"], s["mul_in"],
            s["mul_out"], s["q28_in"], s["q28_out"], s["x"], s["offsets"], s["y"], bias=s["bias"],
            act=c["act"], residual=s["residual"], flags=_flags(c))
    if c["kind"] == "append":
        K.kronq_cache_append(s["k"], s["v"], s["slots"], s["codes"], s["params"],
                             rotate=c["rotate"], k_hat=s["k_hat"], v_hat=s["v_hat"])
        return {"k": s["k_hat"], "v": s["v_hat"], "codes": s["codes"], "params": s["params"]}
    return K.kronq_cache_attention(s["q"], s["codes"], s["params"], s["table"], s["lengths"],
                                   s["starts"], max_new=s["most"], rotate=c["rotate"])


# ---- the definitions in 64 bits -------------------------------------------------------------------
def _sylvester(n):
    """Entry (i, j) of H_n is (-1)^popcount(i & j)."""
    i = torch.arange(n, device=DEV)
    both = i[:, None] & i[None, :]
    odd = torch.zeros_like(both)
    while n > 1:
        odd ^= both & 1
        both >>= 1
        n //= 2
    return (1 - 2 * odd).to(torch.float64)


def _exact_layer(s, e, x):
    """One layer's rows, from the dense matrices of the definition."""
    c = s["case"]

    def of(name):
        v = s[name]
        return v if v is None or c["kind"] != "grouped" else v[e]

    def dense(q28, d):
        if q28 is None:
            return _sylvester(d) / math.sqrt(d)
        return torch.kron(q28.double().contiguous(), _sylvester(d // 28) / math.sqrt(d // 28))

    rows = slice(e * c["d_out"], (e + 1) * c["d_out"])
    words = s["packed"][rows].to(torch.int64) & 0xFFFFFFFF
    words = torch.nn.functional.pad(words, (0, 1))
    j = torch.arange(c["d_in"], device=DEV) * c["bits"]
    codes = ((words[:, j // 32] | words[:, j // 32 + 1] << 32) >> (j % 32)) & (2 ** c["bits"] - 1)
    g = torch.arange(c["d_in"], device=DEV) // c["group"]
    w = s["scales"][rows].double()[:, g] * (codes.double() - s["zeros"][rows].double()[:, g])
    t = x.double() * of("mul_in").double()
    if c["rot_in"]:
        t = t @ dense(of("q28_in"), c["d_in"]).T
    t = t @ w.T
    if c["rot_out"]:
        q28 = of("q28_out")
        t = t @ dense(None if q28 is None else q28.T, c["d_out"]).T
    t = t * of("mul_out").double()
    if s["bias"] is not None:
        t = t + of("bias").double()
    return {"none": lambda z: z, "relu": torch.relu, "silu": torch.nn.functional.silu,
            "gelu": torch.nn.functional.gelu}[c["act"]](t)


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["kind"] == "linear":
        y = _exact_layer(s, 0, s["x"])
        return y if s["residual"] is None else y + s["residual"].double()
    if c["kind"] == "grouped":
        y, at = s["y"].double(), 0
        for e, n in enumerate(_counts(c)):
            if n:
                y[at:at + n] = _exact_layer(s, e, s["x"][at:at + n])
                if s["residual"] is not None:
                    y[at:at + n] += s["residual"][at:at + n].double()
            at += n
        return y
    h = _sylvester(c["dim"]) / math.sqrt(c["dim"])
    if c["kind"] == "append":
        out = {"codes": None, "params": None}
        for name in ("k", "v"):
            r = s[name].double()
            r = r @ h if c["rotate"] else r
            low, high = r.amin(-1, keepdim=True).clamp(max=0), r.amax(-1, keepdim=True).clamp(min=0)
            wide = ((high - low) / 15).clamp(min=MIN_SCALE)
            unit = 2.0 ** (torch.frexp(wide)[1] - 8).double()  # a bf16 step at this size
            scale = torch.ceil(wide / unit) * unit
            zero = torch.round(-low / scale).clamp(max=15)
            out[name] = scale * ((torch.round(r / scale) + zero).clamp(0, 15) - zero)
        return out
    out = []
    group = c["heads"] // c["kv_heads"]
    starts = s["starts"].tolist()
    for b, (length, new) in enumerate(_lengths(c)):
        t = torch.arange(length, device=DEV)
        pages, off = s["table"][b][t // c["page"]].to(torch.int64), t % c["page"]
        d = torch.arange(c["dim"], device=DEV)
        values = []
        for part in (0, 1):
            if part == 0:
                at = off[:, None] * (c["dim"] // 8) + d // 8
            else:
                at = (off[:, None] // 4 * (c["dim"] // 8) + d // 8) * 4 + off[:, None] % 4
            word = s["codes"][pages[:, None], :, part, at].permute(2, 0, 1)
            code = (word >> (4 * (d % 8)).to(torch.int32)) & 15
            param = s["params"][pages, :, part, off].T
            scale = (param & -65536).view(torch.float32).double()[..., None]
            values.append(scale * (code.double() - (param & 0xFFFF).double()[..., None]))
        k, v = (x.repeat_interleave(group, 0) for x in values)
        q = s["q"][starts[b]:starts[b + 1]].double().transpose(0, 1)
        q = q @ h if c["rotate"] else q
        o = torch.empty_like(q)
        for i in range(0, new, 256):
            scores = q[:, i:i + 256] @ k.transpose(1, 2) / math.sqrt(c["dim"])
            last = length - new + torch.arange(i, min(new, i + 256), device=DEV)
            scores = scores.masked_fill(t > last[:, None], -math.inf)
            o[:, i:i + 256] = torch.softmax(scores, -1) @ v
        out.append((o @ h if c["rotate"] else o).transpose(0, 1))
    return torch.cat(out)
