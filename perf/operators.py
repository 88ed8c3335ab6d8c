"""The operators of a serving step of a token model, and what is measured of them: the linear layer in 8-bit integers, the quantised cache of keys
and values with the attention that reads it, and the log probabilities of the tokens that come out.

A case names an operator ("op") and its sizes.  `prepare` makes what a serving program holds before the call; `run` is one call, in plain torch
(in 32 bits) or through `paper_2302_00282_amd.tokens`; `exact` is the definition in 64 bits."""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5                   # of the norm in front of a linear layer
TINY = 2.0 ** -100           # the smallest amplitude of a quantised row


def _linear(m, k, n, dtype="bf16", *, norm=False, bias=False, residual=False, relu=False):
    return dict(op="linear", m=m, k=k, n=n, dtype=dtype, norm=norm, bias=bias, residual=residual, relu=relu)


def _cache(seqs, new, history, heads, dim, page, dtype="bf16"):
    return dict(op="cache", seqs=seqs, new=new, history=history, heads=heads, dim=dim, page=page, dtype=dtype)


def _attention(seqs, queries, longest, heads, kv_heads, dim, page, *, prefix=0, ragged=True):
    return dict(op="attention", seqs=seqs, queries=queries, longest=longest, heads=heads, kv_heads=kv_heads, dim=dim, page=page, prefix=prefix, ragged=ragged)


def _logprobs(rows, vocab, top, dtype="f32", *, pad=0):
    return dict(op="logprobs", rows=rows, vocab=vocab, top=top, dtype=dtype, pad=pad)


def listed():
    return [
        # one token through the first product of a small feed-forward block: the least a linear layer can be asked, all latency
        dict(_linear(1, 512, 2048, norm=True, relu=True), name="linear_1x512x2048_bf16"),
        # a server batch through a wide classifier's first layer: the weights are the work
        dict(_linear(32, 25088, 4096, bias=True, relu=True), name="linear_32x25088x4096_bf16"),
        # a prompt of odd length through a layer of odd sizes, with the block's shortcut, in fp32
        dict(_linear(517, 1001, 1003, "f32", norm=True, bias=True, residual=True), name="linear_517x1001x1003_f32"),
        # many prompts at once: the products are the work
        dict(_linear(8192, 8192, 8192), name="linear_8192x8192x8192_bf16"),
        # one more token of each of four short dialogues, and their whole past read back
        dict(_cache(4, 1, 33, 8, 64, 16), name="cache_4x1_of_33_bf16"),
        # prompts written and read back, heads of an odd width, as one product wrote them: strided rows
        dict(_cache(7, 1171, 1171, 10, 80, 48, "f32"), name="cache_7x1171_f32"),
        # the next token of one short dialogue: all latency
        dict(_attention(1, 1, 37, 8, 8, 64, 16), name="attention_1_of_37"),
        # the next token of sixteen long dialogues of unequal length
        dict(_attention(16, 1, 32768, 32, 8, 128, 64), name="attention_16_of_32768"),
        # the next token of 64 dialogues that begin with the same long instructions
        dict(_attention(64, 1, 500, 32, 4, 128, 64, prefix=16384), name="attention_64_prefix_16384"),
        # a whole prompt, every token seeing those before it
        dict(_attention(1, 4097, 4097, 20, 4, 128, 32, ragged=False), name="attention_prompt_4097"),
        # the choice of one next token
        dict(_logprobs(1, 32000, 5), name="logprobs_1x32000_f32"),
        # prompts scored token by token, rows of an odd length with some columns behind them
        dict(_logprobs(2048, 100003, 20, "bf16", pad=61), name="logprobs_2048x100003_bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Any of the operators: one token to thousands, sizes even and odd, both types where the operator has two, heads shared and not, pages of 16 to 256 tokens."""
    op = rng.choice(["linear", "cache", "attention", "attention", "logprobs"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "linear":
        m, k, n = _log(rng, 1, 8192), _log(rng, 64, 25088), _log(rng, 64, 16384)
        if rng.random() < 0.5:
            k, n = -(-k // 64) * 64, -(-n // 64) * 64
        return _linear(min(m, max(1, 8192 ** 3 // (k * n))), k, n, dtype, **{o: rng.random() < 0.4 for o in ("norm", "bias", "residual", "relu")})
    heads, dim, page = rng.choice([1, 2, 4, 5, 8, 16]), rng.choice([32, 64, 64, 80, 96, 128, 128, 192, 256]), rng.choice([16, 32, 48, 64, 128, 256])
    if op == "cache":
        seqs, new = _log(rng, 1, 64), rng.choice([1, _log(rng, 1, 4096)])
        history = new + rng.choice([0, _log(rng, 1, 4096)])
        cut = max(1, seqs * history * heads * dim * 2 // (16 << 20))
        return _cache(max(1, seqs // cut), new, history, heads, dim, page, dtype)
    if op == "attention":
        group = rng.choice([1, 1, 2, 3, 4, 5, 8, 16])
        queries = rng.choice([1, 1, 1, _log(rng, 2, 8), _log(rng, 8, 2048)])
        seqs, longest = _log(rng, 1, 128), max(queries, _log(rng, 1, 32768))
        prefix = rng.choice([0, 0, _log(rng, 16, 32768)])
        seqs = max(1, min(seqs, (1 << 29) // (longest * heads * dim)))                             # (keys of the sequences)
        seqs = max(1, min(seqs, (1 << 29) // (queries * heads * group * (longest + prefix))))      # (and products of queries with keys)
        while queries * heads * group * (longest + prefix) > 1 << 29:
            queries = max(1, queries // 2)
            longest = max(queries, longest // 2)
        return _attention(seqs, queries, longest, heads * group, heads, dim, page, prefix=prefix, ragged=rng.random() < 0.7)
    vocab = _log(rng, 1000, 200000)
    return _logprobs(_log(rng, 1, min(4096, (3 << 26) // vocab)), vocab, rng.choice([0, 1, 5, 20, 32]), dtype, pad=rng.choice([0, 0, rng.randint(1, 64)]))


# ---- what a serving program holds before the call -----------------------------------------------------------------------------------------


class _Draws:
    def __init__(self, seed):
        self.host = random.Random(seed)
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)

    def normal(self, *shape, std=1.0):
        return torch.randn(shape, generator=self.gen, device="cuda").mul_(std)

    def uniform(self, *shape, lo=0.0, hi=1.0):
        return torch.rand(shape, generator=self.gen, device="cuda").mul_(hi - lo).add_(lo)

    def whole(self, lo, hi, *shape, dtype=torch.int32):
        return torch.randint(lo, hi, shape, generator=self.gen, device="cuda", dtype=dtype)

    def order(self, n):
        return torch.randperm(n, generator=self.gen, device="cuda")


def _pitch(k):
    """Bytes from one quantised row to the next: a multiple of 128, zeros behind the row's own."""
    return -(-k // 128) * 128


def _prepare_linear(c, d):
    m, k, n, t = c["m"], c["k"], c["n"], TYPES[c["dtype"]]
    w = torch.zeros(n, _pitch(k), dtype=torch.int8, device="cuda")
    w[:, :k] = d.whole(-127, 128, n, k, dtype=torch.int8)
    x = d.normal(m, k)
    x[:, :: max(1, k // 7)] *= 6.0                                            # (a few channels are far larger than the rest)
    return dict(x=x.to(t), w=w, w_scale=d.uniform(n, lo=0.5, hi=1.5).div_(73.0 * math.sqrt(k)),
                gamma=d.uniform(k, lo=0.5, hi=1.5) if c["norm"] else None, bias=d.normal(n, std=0.1) if c["bias"] else None,
                residual=d.normal(m, n).to(t) if c["residual"] else None)


def _pages(c, lengths, d, shared=0):
    """A pool of pages in no order, the table of each sequence's pages, and the pages of the shared prefix."""
    page = c["page"]
    per = [-(-x // page) for x in lengths]
    most, before = max(per), -(-shared // page)
    order = d.order(before + sum(per) + 3).to(torch.int32)
    tables = torch.zeros(len(per), most, dtype=torch.int32, device="cuda")
    at = before
    for b, p in enumerate(per):
        tables[b, :p] = order[at:at + p]
        at += p
    return len(order), tables, order[:before]


def _pool(c, n, heads, d):
    """A cache of n pages filled with what quantised rows hold: amplitudes up to 127, a scale for each token and head."""
    page, dim = c["page"], c["dim"]
    return dict(k=d.whole(-127, 128, n, heads, page, dim, dtype=torch.int8), v=d.whole(-127, 128, n, heads, page // 16, dim, 16, dtype=torch.int8),
                k_scale=d.uniform(n, heads, page, lo=0.5, hi=1.5).div_(73.0), v_scale=d.uniform(n, heads, page, lo=0.5, hi=1.5).div_(73.0))


def _prepare_cache(c, d):
    b, new, history, heads, dim, page, t = c["seqs"], c["new"], c["history"], c["heads"], c["dim"], c["page"], TYPES[c["dtype"]]
    n, tables, _ = _pages(c, [history] * b, d)
    at = torch.arange(history, device="cuda")
    slots = tables.long()[:, at // page] * page + at % page                   # [sequence][token]
    kv = d.normal(b * new, 2, heads, dim).to(t)                               # (as one product writes them: keys and values of a token side by side)
    return dict(_pool(c, n, heads, d), new_k=kv[:, 0], new_v=kv[:, 1], write=slots[:, history - new:].reshape(-1).contiguous(), read=slots.reshape(-1).contiguous())


def _lengths(c, seed):
    """Tokens of each sequence, and how many of them, the last ones, are the queries."""
    rng = random.Random(seed)
    b, q, most = c["seqs"], c["queries"], c["longest"]
    if not c["ragged"]:
        return [most] * b, [q] * b
    queries = [q] + [rng.randint(1, q) for _ in range(b - 1)]
    return [most] + [rng.randint(x, most) for x in queries[1:]], queries


def _prepare_attention(c, d, seed):
    lengths, queries = _lengths(c, seed)
    n, tables, prefix = _pages(c, lengths, d, c["prefix"])
    starts = [0]
    for q in queries:
        starts.append(starts[-1] + q)
    return dict(_pool(c, n, c["kv_heads"], d), q=d.normal(starts[-1], c["heads"], c["dim"]).to(torch.bfloat16), tables=tables, prefix_table=prefix,
                lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"), starts=torch.tensor(starts, dtype=torch.int32, device="cuda"),
                max_queries=max(queries), max_length=max(lengths))


def _prepare_logprobs(c, d):
    rows, vocab = c["rows"], c["vocab"]
    logits = torch.empty(rows, vocab + c["pad"], dtype=TYPES[c["dtype"]], device="cuda")
    for part in logits.split(256):
        part.copy_(d.normal(*part.shape, std=2.5))
    likely = d.whole(0, vocab, rows, 4, dtype=torch.int64)
    logits.scatter_(1, likely, d.uniform(rows, 4, lo=8.0, hi=20.0).to(logits.dtype))     # (a model is fairly sure of a few tokens)
    logits[:, d.whole(0, vocab, max(1, vocab // 500), dtype=torch.int64)] = -math.inf      # (some may not be said at all)
    targets = torch.where(d.uniform(rows) < 0.7, likely[:, 0], d.whole(0, vocab, rows, dtype=torch.int64))
    targets[d.uniform(rows) < 0.05] = -1                                                 # (and some positions have none)
    return dict(logits=logits[:, :vocab], targets=targets)


def prepare(case, seed):
    d = _Draws(seed)
    op = case["op"]
    state = (_prepare_linear(case, d) if op == "linear" else _prepare_cache(case, d) if op == "cache" else
             _prepare_attention(case, d, seed) if op == "attention" else _prepare_logprobs(case, d))
    return dict(state, case=case)


# ---- the plain forms -------------------------------------------------------------------------------------------------------------------------


def _quantized(x):
    """Rows of x as whole numbers up to 127 (held in 32 bits) and their scales."""
    a = x.abs().amax(-1, keepdim=True).clamp_min(TINY)
    full = torch.full_like(a, 127.0)
    return torch.round(x * torch.div(full, a)), torch.div(a, full)


def _plain_linear(s):
    c, x = s["case"], s["x"].float()
    q, scale = _quantized(x * s["gamma"] if c["norm"] else x)
    if c["norm"]:
        scale = scale * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    y = (q @ s["w"][:, :c["k"]].float().t()) * scale * s["w_scale"]
    if c["bias"]:
        y = y + s["bias"]
    if c["residual"]:
        y = y + s["residual"].float()
    return (y.clamp_min(0) if c["relu"] else y).to(s["x"].dtype)


def _plain_cache(s):
    page, t = s["case"]["page"], s["new_k"].dtype
    for_k, for_v = s["k"], s["v"]
    at, tok = s["write"] // page, s["write"] % page
    qk, sk = _quantized(s["new_k"].float())
    qv, sv = _quantized(s["new_v"].float())
    for_k[at, :, tok] = qk.to(torch.int8)
    for_v[at, :, tok // 16, :, tok % 16] = qv.to(torch.int8)
    s["k_scale"][at, :, tok], s["v_scale"][at, :, tok] = sk.squeeze(-1), sv.squeeze(-1)
    at, tok = s["read"] // page, s["read"] % page
    k = for_k[at, :, tok].float() * s["k_scale"][at, :, tok].unsqueeze(-1)
    v = for_v[at, :, tok // 16, :, tok % 16].float() * s["v_scale"][at, :, tok].unsqueeze(-1)
    return k.to(t), v.to(t)


def _gathered(s, pages):
    """Keys and values of rows of pages in 32 bits: [row][head][token][dim]."""
    b, n = pages.shape
    _, h, page, dim = s["k"].shape
    k = s["k"][pages].permute(0, 2, 1, 3, 4).float() * s["k_scale"][pages].permute(0, 2, 1, 3).unsqueeze(-1)
    v = s["v"][pages].permute(0, 2, 1, 3, 5, 4).reshape(b, h, n, page, dim).float() * s["v_scale"][pages].permute(0, 2, 1, 3).unsqueeze(-1)
    return k.reshape(b, h, n * page, dim), v.reshape(b, h, n * page, dim)


def _plain_attention(s):
    c, q = s["case"], s["q"].float()
    h, g, dim, most = c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"], s["max_queries"]
    starts, lengths = s["starts"].long(), s["lengths"].long()
    b, counts = len(lengths), starts[1:] - starts[:-1]
    i = torch.arange(most, device="cuda")
    rows = (starts[:-1, None] + i).clamp_max(len(q) - 1)                                   # [sequence][query]
    qs = q[rows].view(b, most, h, g, dim).permute(0, 2, 3, 1, 4).reshape(b, h, g * most, dim) / math.sqrt(dim)
    k, v = _gathered(s, s["tables"].long())
    j = torch.arange(k.shape[2], device="cuda")
    seen = (j < (lengths - counts)[:, None, None] + i[:, None] + 1)[:, None, None]         # [sequence][1][1][query][key]
    scores = torch.matmul(qs, k.transpose(2, 3).contiguous()).view(b, h, g, most, -1).masked_fill(~seen, -math.inf).view(b, h, g * most, -1)
    if c["prefix"]:
        pk, pv = _gathered(s, s["prefix_table"].long()[None])
        pk, pv = pk[0, :, :c["prefix"]], pv[0, :, :c["prefix"]]
        together = qs.transpose(0, 1).reshape(h, -1, dim)                                  # (the rows of all sequences against the one prefix)
        before = torch.matmul(together, pk.transpose(1, 2).contiguous()).view(h, b, g * most, -1).transpose(0, 1)
        scores = torch.cat([before, scores], -1)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p[..., c["prefix"]:], v)
    if c["prefix"]:
        before = p[..., :c["prefix"]].transpose(0, 1).reshape(h, b * g * most, -1)
        out = out + torch.matmul(before, pv).view(h, b, g * most, dim).transpose(0, 1)
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    out = out.view(b, h, g, most, dim).permute(0, 3, 1, 2, 4).reshape(b, most, h * g, dim)
    return out[i < counts[:, None]].to(s["q"].dtype)


def _plain_logprobs(s):
    top, targets, x = s["case"]["top"], s["targets"], s["logits"].float()
    m = x.amax(-1, keepdim=True)
    below = x - m
    e = torch.exp(below)
    total = e.sum(-1, keepdim=True)
    entropy = torch.log(total) - torch.where(e > 0, below * e, torch.zeros_like(e)).sum(-1, keepdim=True) / total
    lse = m + torch.log(total)
    given = (x.gather(1, targets.clamp_min(0)[:, None]) - lse).squeeze(1)
    best, index = torch.sort(x, dim=1, descending=True, stable=True)
    return torch.where(targets >= 0, given, torch.zeros_like(given)), entropy.squeeze(1), best[:, :top] - lse, index[:, :top].to(torch.int32)


def _own(s):
    from paper_2302_00282_amd import tokens as T
    c = s["case"]
    if c["op"] == "linear":
        return T.linear(s["x"], s["w"], s["w_scale"], bias=s["bias"], residual=s["residual"], relu=c["relu"], gamma=s["gamma"], eps=EPS)
    if c["op"] == "logprobs":
        return T.logprobs(s["logits"], s["targets"], top=c["top"])
    cache = T.KVCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
    if c["op"] == "cache":
        cache.write(s["new_k"], s["new_v"], s["write"])
        return cache.read(s["read"], s["new_k"].dtype)
    return T.attention(s["q"], cache, s["tables"], s["lengths"], starts=s["starts"], max_queries=s["max_queries"], max_length=s["max_length"],
                       prefix_table=s["prefix_table"] if c["prefix"] else None, prefix_length=c["prefix"])


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    return (_plain_linear(state) if op == "linear" else _plain_cache(state) if op == "cache" else
            _plain_attention(state) if op == "attention" else _plain_logprobs(state))


# ---- the least that has to be done, and the definitions in 64 bits ---------------------------------------------------------------------------


def work(case):
    c = case
    b = 2 if c.get("dtype", "bf16") == "bf16" else 4
    if c["op"] == "linear":
        m, k, n = c["m"], c["k"], c["n"]
        return {"bytes": b * (m * k + m * n * (2 if c["residual"] else 1)) + n * k + 4 * n * (2 if c["bias"] else 1) + (4 * k if c["norm"] else 0), "flops": 2 * m * n * k}
    if c["op"] == "cache":
        rows, past = c["seqs"] * c["new"] * c["heads"] * 2, c["seqs"] * c["history"] * c["heads"] * 2
        return {"bytes": (rows + past) * (c["dim"] * (b + 1) + 4), "flops": 4 * (rows + past) * c["dim"]}
    if c["op"] == "logprobs":
        n = c["rows"] * c["vocab"]
        return {"bytes": n * b + c["rows"] * (16 + 8 * c["top"]), "flops": 6 * n}
    lengths, queries = _lengths(c, 1)
    pairs = sum(q * c["prefix"] + q * n - q * (q - 1) // 2 for n, q in zip(lengths, queries))
    keys = sum(lengths) + c["prefix"]
    return {"bytes": keys * c["kv_heads"] * 2 * (c["dim"] + 4) + 4 * sum(queries) * c["heads"] * c["dim"], "flops": 4 * pairs * c["heads"] * c["dim"]}


def _exact_rows(x):
    a = x.abs().amax(-1, keepdim=True).clamp_min(TINY)
    return torch.round(x * 127.0 / a), a / 127.0


def _exact_linear(s, c):
    parts = []
    w = s["w"][:, :c["k"]].double()
    for r in range(0, c["m"], 2048):
        x = s["x"][r:r + 2048].double()
        q, scale = _exact_rows(x * s["gamma"].double() if c["norm"] else x)
        if c["norm"]:
            scale = scale / torch.sqrt(torch.mean(x * x, -1, keepdim=True) + EPS)
        y = torch.matmul(q, w.t()) * scale * s["w_scale"].double()
        if c["bias"]:
            y += s["bias"].double()
        if c["residual"]:
            y += s["residual"][r:r + 2048].double()
        parts.append(torch.relu(y) if c["relu"] else y)
    return torch.cat(parts)


def _exact_cache(s, c):
    """Row by row of what was written, by the slots' order; the past as it lies there."""
    out = []
    for new, held, scale, is_v in ((s["new_k"], s["k"], s["k_scale"], False), (s["new_v"], s["v"], s["v_scale"], True)):
        n, h, page, dim = s["k"].shape
        rows = held.transpose(3, 4).reshape(n, h, page, dim) if is_v else held
        rows = (rows.double() * scale.double()[..., None]).transpose(1, 2).reshape(n * page, h, dim)
        q, a = _exact_rows(new.double())
        rows[s["write"]] = q * a
        out.append(rows[s["read"]])
    return tuple(out)


def _exact_attention(s, c, seed):
    lengths, queries = _lengths(c, seed)
    page, h, g, dim, prefix = c["page"], c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"], c["prefix"]

    def tokens(table, n, head):
        at = torch.arange(n, device="cuda")
        p, t = table.long()[at // page], at % page
        return s["k"][p, head, t].double() * s["k_scale"][p, head, t].double()[:, None], s["v"][p, head, t // 16, :, t % 16].double() * s["v_scale"][p, head, t].double()[:, None]

    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for head in range(h):
        front = tokens(s["prefix_table"], prefix, head) if prefix else None
        first = 0
        for b, (n, m) in enumerate(zip(lengths, queries)):
            k, v = tokens(s["tables"][b], n, head)
            if prefix:
                k, v = torch.cat([front[0], k]), torch.cat([front[1], v])
            hidden = torch.arange(n + prefix, device="cuda")[None, :] > prefix + n - m + torch.arange(m, device="cuda")[:, None]
            for j in range(head * g, head * g + g):
                x = s["q"][first:first + m, j].double() @ k.t() / math.sqrt(dim)
                out[first:first + m, j] = torch.softmax(x.masked_fill(hidden, -math.inf), -1) @ v
            first += m
    return out


def _exact_logprobs(s, c):
    parts = []
    for x, t in zip(s["logits"].split(64), s["targets"].split(64)):
        lp = torch.log_softmax(x.double(), -1)
        given = torch.where(t >= 0, lp.gather(1, t.clamp_min(0)[:, None])[:, 0], 0.0)
        parts.append((given, -torch.nan_to_num(lp.exp() * lp, nan=0.0).sum(-1), torch.sort(lp, 1, True).values[:, :c["top"]]))
    return tuple(torch.cat(p) for p in zip(*parts)) + (None,)


def exact(case, seed):
    s = prepare(case, seed)
    return (_exact_linear(s, case) if case["op"] == "linear" else _exact_cache(s, case) if case["op"] == "cache" else
            _exact_attention(s, case, seed) if case["op"] == "attention" else _exact_logprobs(s, case))
