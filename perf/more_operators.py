"""The 8-bit paged key/value cache and attention with shared prefixes, as timed cases with their plain forms and a 64-bit reference.

Requests keep their keys and values in pages of a shared pool.  Four operators:

append     normalises and rotates the new tokens' keys and stores keys and values as e4m3 codes with a power of two per token and head as their scale;
           what was stored is read back, so that it can be looked at.
read       brings the keys and values of given places back, as rows.
attention  lets the new tokens' queries attend to their request's keys in an 8-bit cache, each up to its own position.
shared     the same where groups of requests start with the same pages (a system prompt, a document that many ask about): the keys and values that a
           group shares are read once for all of its rows.  One plan a step serves all of a model's layers.

A case names the operator, the head layout, the cache's type, the page size and what the requests bring: `requests` of them, each with up to `cached` tokens of
its own in the cache already; the first `chunks` of them bring up to `new` tokens, the others one.  Where `ragged` is set the lengths differ, some requests hold
nothing of their own yet and some bring nothing.  `groups` of shared prefixes of up to `prefix` tokens, in whole pages, stand in front of the requests in no
particular order; where ragged, some requests belong to none.  Lengths follow from the case; values, page numbers and their order from the seed.

The rows of the fused projection are fp32 [rows, (query heads + 2 key/value heads) * head dim].  Room for rows is rounded up to 16; what lies behind the last
row stays as it was.
"""
import math
import random

import numpy as np
import torch

own = False

EPS, THETA = 1e-6, 1e6
E4M3_MAX = 448.0
LEAST_SCALE = 16      # biased exponent: 2^-111

# head layouts of the models that the benchmark and the tests run
_TINY = dict(q_heads=4, kv_heads=2, head_dim=64)
_H16 = dict(q_heads=16, kv_heads=8, head_dim=128)
_H32 = dict(q_heads=32, kv_heads=8, head_dim=128)
_H14 = dict(q_heads=14, kv_heads=2, head_dim=64)
_H12 = dict(q_heads=12, kv_heads=2, head_dim=128)

_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
_BYTES = {"bf16": 2, "fp32": 4, "e4m3": 1}


def _case(name, op, heads, **kw):
    c = dict(op=op, dtype="e4m3", page=64, requests=1, cached=0, new=1, chunks=0, groups=0, prefix=0, layers=1, ragged=False, mix=0, **heads)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one user's next token
        _case("append, one token", "append", _H32, cached=1024),
        # prompts of several users cut to one step's room
        _case("append, prompts", "append", _H32, page=32, requests=3, cached=700, new=900, chunks=3, ragged=True, mix=7),
        # a request moves to another place: its tokens come out of the pool
        _case("read, 1000 tokens", "read", _H16, page=16, cached=1000),
        # a batch is swapped out
        _case("read, 16 ragged", "read", _H32, page=32, requests=16, cached=8000, ragged=True, mix=3),
        # the benchmark's own configuration: one user, 1024 tokens in the cache
        _case("decode 1 x 1024", "attention", _H32, cached=1024),
        # the batched configuration, at lengths as they are in a running server
        _case("decode 32, ragged", "attention", _H32, page=16, requests=32, cached=2304, ragged=True, mix=5),
        # long contexts, two tokens that wait for their refill and the newest one
        _case("3 rows, 8 x 16k", "attention", _H32, page=128, requests=8, cached=16384, new=3, chunks=8),
        # the last part of a prompt of 8192
        _case("2048 rows behind 6144", "attention", _H32, cached=6144, new=2048, chunks=1),
        # a full server behind one system prompt
        _case("64 behind 4096", "shared", _H32, dtype="bf16", requests=64, cached=400, groups=1, prefix=4096, layers=4, ragged=True, mix=11),
        # several documents, questions about each, 8-bit
        _case("4 documents, 48 askers", "shared", _H16, page=32, requests=48, cached=300, new=3, chunks=48, groups=4, prefix=8192, layers=4, ragged=True, mix=12),
        # new questions arrive at one document, beside answers that go on
        _case("chunks behind a document", "shared", _H14, dtype="bf16", page=32, requests=12, cached=200, new=120, chunks=6, groups=1, prefix=10000, layers=2, ragged=True, mix=13),
        # the tiny model of the parity tests
        _case("tiny fp32, shared", "shared", _TINY, dtype="fp32", page=16, requests=6, cached=40, new=4, chunks=2, groups=2, prefix=200, layers=1, ragged=True, mix=14),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["append", "read", "attention", "attention", "shared", "shared", "shared"])
        c = _case("", op, rng.choice([_TINY, _H16, _H32, _H32, _H14, _H12]), page=rng.choice([16, 32, 64, 128, 256]))
        c.update(requests=_log(rng, 1, 64), cached=_log(rng, 1, 16384 if op != "shared" else 2048) - 1, ragged=rng.random() < 0.7, mix=rng.randrange(1 << 20))
        if rng.random() < 0.6 and op != "read":
            c.update(new=_log(rng, 2, 2048), chunks=rng.randint(1, c["requests"]))
        if op == "shared":
            c.update(dtype=rng.choice(["bf16", "bf16", "e4m3"]), groups=_log(rng, 1, 8), prefix=_log(rng, 16, 16384), layers=rng.choice([1, 2, 4]))
        if op == "read":
            c.update(dtype=rng.choice(["e4m3", "e4m3", "bf16", "fp32"]))
        if op == "shared" and rng.random() < 0.15:      # the fp32 models are small ones
            c.update(dtype="fp32", cached=min(c["cached"], 500), new=min(c["new"], 64), prefix=min(c["prefix"], 2048))
        w = _layout(c)
        keys = len(w["start"]) * max(s + r for s, r in zip(w["start"], w["rows"]))
        if op != "read" and sum(w["rows"]) > 4096:
            continue
        # the plain form pads requests and rows to the longest: its scores and its copies of the cache
        if max(keys * max(w["rows"]) * c["q_heads"], 2 * keys * c["kv_heads"] * c["head_dim"]) > 2 << 30:
            continue
        if (sum(w["start"]) if op == "read" else sum(w["rows"])) > 0 and _cost(c) <= most:
            return c


def _layout(c):
    """Tokens in the cache and new tokens of each request, its group or -1, and the groups' pages."""
    rng = random.Random(c["mix"])
    pages = []
    for _ in range(c["groups"]):
        p = _log(rng, max(1, c["prefix"] // 4), c["prefix"]) if c["ragged"] and c["groups"] > 1 else c["prefix"]
        pages.append(max(1, p // c["page"]))
    start, rows, group = [], [], []
    for i in range(c["requests"]):
        s, r = c["cached"], c["new"] if i < c["chunks"] else 1
        if c["ragged"]:
            s = 0 if rng.random() < 0.1 else _log(rng, max(1, s // 16), s + 1) - 1
            r = 0 if c["requests"] > 3 and rng.random() < 0.06 else rng.randint((r + 1) // 2, r)
        g = rng.randrange(c["groups"]) if c["groups"] else -1
        if c["ragged"] and rng.random() < 0.08:
            g = -1
        start.append(s + (pages[g] * c["page"] if g >= 0 else 0))
        rows.append(0 if c["op"] == "read" else r)
        group.append(g)
    if sum(rows) == 0 and c["op"] != "read":
        rows[0] = 1
    return dict(start=start, rows=rows, group=group, pages=pages)


def _cost(c):
    w = work(c)
    return w["bytes"] / 2.5e12 + w["flops"] / (2e13 if c["dtype"] == "fp32" else 5e14) + 1e-5


def work(c):
    w = _layout(c)
    start, rows = w["start"], w["rows"]
    n, hd, nkv, nq = sum(rows), c["head_dim"], c["kv_heads"], c["q_heads"]
    row = hd * _BYTES[c["dtype"]] + (1 if c["dtype"] == "e4m3" else 0)      # of one head's key or value in the cache, with its scale
    if c["op"] == "append":       # a row's key and value in and out, its angles; and read back
        return {"bytes": n * (2 * nkv * (4 * hd + row) + 4 * hd) + n * 2 * nkv * (row + 2 * hd), "flops": n * nkv * hd * 8}
    if c["op"] == "read":
        return {"bytes": sum(start) * (2 * nkv * (row + hd * (4 if c["dtype"] == "fp32" else 2)) + 8), "flops": 0}
    live = [(s, r, g) for s, r, g in zip(start, rows, w["group"]) if r]
    keys = sum(s + r - (w["pages"][g] * c["page"] if g >= 0 else 0) for s, r, g in live) + sum(w["pages"][g] * c["page"] for g in {g for _, _, g in live if g >= 0})
    seen = sum(r * s + r * (r + 1) // 2 for s, r, _ in live)
    return {"bytes": c["layers"] * (2 * keys * nkv * row + n * nq * hd * (4 + (4 if c["dtype"] == "fp32" else 2))), "flops": c["layers"] * 4 * seen * nq * hd}


# ------------------------------------------------------------------------------------------------ e4m3 rows with a power of two as their scale

def _power(e):
    """2^(e - 127) of biased exponents 1 .. 254."""
    return (e.int() << 23).view(torch.float32)


def _to_codes(x):
    """Codes of fp32 rows [..., head dim] and the biased exponents [...] of their scales: the least power of two that brings the row's largest magnitude to at most 448."""
    most = x.abs().amax(-1)
    frac, exp = torch.frexp(most / E4M3_MAX)                      # most / 448 = frac 2^exp, 0.5 <= frac < 1
    e = torch.where(frac == 0.5, exp - 1, exp) + 127
    e = torch.where(most > 0, e, LEAST_SCALE).clamp(min=LEAST_SCALE)
    return (x * _power(254 - e).unsqueeze(-1)).to(torch.float8_e4m3fn), e.to(torch.uint8)


def _values(codes, scales):
    """fp32 values that codes (as bytes) [..., head dim] and scales [...] stand for."""
    return codes.view(torch.float8_e4m3fn).float() * _power(scales).unsqueeze(-1)


# ------------------------------------------------------------------------------------------------ inputs

def prepare(c, seed):
    w = _layout(c)
    start, rows, group = w["start"], w["rows"], w["group"]
    page, hd, nkv, total, dt = c["page"], c["head_dim"], c["kv_heads"], sum(rows), _TYPES[c["dtype"]]
    room = max(16, -(-total // 16) * 16)
    ends = [-(-(s + r) // page) for s, r in zip(start, rows)]
    front = [w["pages"][g] if g >= 0 else 0 for g in group]
    width = max(ends) + 1
    n_pages = sum(w["pages"]) + sum(ends) - sum(front) + 7
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    order = np.random.RandomState(seed % (1 << 31)).permutation(n_pages).astype(np.int32)
    table = np.full((len(start), width), -1, np.int32)
    at, prefixes = 0, []
    for p in w["pages"]:
        prefixes.append(order[at:at + p])
        at += p
    for i, (e, f, g) in enumerate(zip(ends, front, group)):
        if f:
            table[i, :f] = prefixes[g]
        table[i, f:e] = order[at:at + e - f]
        at += e - f

    def ints(a, t=torch.int32):
        return torch.as_tensor(np.asarray(a), dtype=t).to("cuda")

    def normal(*shape, mean=0.0, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32) * std + mean).to(dtype)

    def pool():
        x = normal(n_pages, nkv, page, hd, std=math.exp(np.random.RandomState(seed % 977).uniform(-1, 1)))
        return _to_codes(x) if c["dtype"] == "e4m3" else (x.to(dt), None)

    s = dict(op=c["op"], page=page, q_heads=c["q_heads"], kv_heads=nkv, head_dim=hd, dtype=dt, total=total, longest=max(a + b for a, b in zip(start, rows)),
             most_rows=max(rows), room=room, table=ints(table), start=ints(start), rows=ints(rows))
    s["layers"] = [pool() + pool() for _ in range(c["layers"])]      # codes or values of the keys, their scales, the values', theirs
    wide = torch.float32 if c["dtype"] == "fp32" else torch.bfloat16
    if c["op"] == "read":
        places = np.concatenate([table[i, np.arange(n) // page].astype(np.int64) * page + np.arange(n) % page for i, n in enumerate(start)])
        s["places"] = ints(places, torch.int64)
        s["k_rows"], s["v_rows"] = (torch.zeros(len(places), nkv, hd, device="cuda", dtype=wide) for _ in range(2))
        return s
    positions = np.concatenate([np.arange(a, a + b) for a, b in zip(start, rows)])
    owner = np.repeat(np.arange(len(rows)), rows)
    places = table[owner, positions // page].astype(np.int64) * page + positions % page
    behind = np.full(room - total, -1)
    s.update(cu=ints(np.concatenate([[0], np.cumsum(rows)])), pos=ints(np.concatenate([positions, behind])), places=ints(np.concatenate([places, behind]), torch.int64))
    s["qkv"] = normal(room, (c["q_heads"] + 2 * nkv) * hd)
    s["gain"] = normal(hd, mean=1.0, std=0.2, dtype=wide)
    angle = torch.arange(width * page, device="cuda", dtype=torch.float64)[:, None] * THETA ** (-torch.arange(0, hd, 2, device="cuda", dtype=torch.float64) / hd)
    s["rope"] = torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()      # [positions, head dim / 2, (cos, sin)]
    if c["op"] == "append":
        s["k_rows"], s["v_rows"] = (torch.zeros(room, nkv, hd, device="cuda", dtype=wide) for _ in range(2))
    else:
        s["out"] = [torch.zeros(room, c["q_heads"], hd, device="cuda", dtype=wide) for _ in range(c["layers"])]
    if c["op"] == "shared":
        s["group"] = ints(group)
        s["prefix_pages"] = ints(w["pages"])
    return s


# ------------------------------------------------------------------------------------------------ the framework's operators

def _handles(s):
    """The layers' handles and the plan's buffers, which a program keeps for as long as it keeps the pools."""
    if "handles" not in s:
        import paper_2510_11958_amd as pkg
        k, ks, v, vs = s["layers"][0]
        first = pkg.PagedCache(k, v, s["table"], n_q_heads=s["q_heads"], max_rows=s["room"], k_scale=ks, v_scale=vs)
        s["handles"] = [first] + [first.layer(k, v, k_scale=ks, v_scale=vs) for k, ks, v, vs in s["layers"][1:]]
        if s["op"] == "shared":
            s["plan"] = pkg.SharedPlan(first, n_groups=s["prefix_pages"].numel())
    return s["handles"]


def _own(s):
    handles = _handles(s)
    if s["op"] == "append":
        handles[0].append(s["qkv"], s["cu"], s["pos"], s["places"], k_norm=s["gain"], rope=s["rope"], eps=EPS)
    if s["op"] in ("append", "read"):
        handles[0].read(s["places"], s["k_rows"], s["v_rows"])
    elif s["op"] == "attention":
        handles[0].attention(s["qkv"], s["start"], s["cu"], s["out"][0], q_norm=s["gain"], rope=s["rope"], eps=EPS, max_new=s["most_rows"])
    else:
        s["plan"].build(s["start"], s["cu"], s["group"], s["prefix_pages"])
        for cache, out in zip(handles, s["out"]):
            cache.attention_shared(s["plan"], s["qkv"], out, q_norm=s["gain"], rope=s["rope"], eps=EPS)


# ------------------------------------------------------------------------------------------------ plain forms

def _norm_rotate(x, gain, rope, pos):
    """x fp32 [..., heads, head dim] at positions pos [...]: RMS norm with gain, then the rotation of the pairs (i, i + head dim / 2)."""
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.float()
    a, b = x.chunk(2, -1)
    cos, sin = rope[pos].unsqueeze(-3).unbind(-1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _append(s):
    n, hd, nq, nkv, page = s["total"], s["head_dim"], s["q_heads"], s["kv_heads"], s["page"]
    x = s["qkv"][:n].view(n, nq + 2 * nkv, hd)
    at = s["places"][:n]
    k, ks, v, vs = s["layers"][0]
    key, key_scale = _to_codes(_norm_rotate(x[:, nq:nq + nkv], s["gain"], s["rope"], s["pos"][:n].long()))
    value, value_scale = _to_codes(x[:, nq + nkv:])
    k.view(torch.uint8)[at // page, :, at % page] = key.view(torch.uint8)
    v.view(torch.uint8)[at // page, :, at % page] = value.view(torch.uint8)
    ks[at // page, :, at % page] = key_scale
    vs[at // page, :, at % page] = value_scale


def _rows_at(s, x, scale, at):
    page = s["page"]
    if scale is None:
        return x[at // page, :, at % page]
    return _values(x.view(torch.uint8)[at // page, :, at % page], scale[at // page, :, at % page])


def _read(s, n):
    k, ks, v, vs = s["layers"][0]
    at = s["places"][:n]
    s["k_rows"][:n] = _rows_at(s, k, ks, at).to(s["k_rows"].dtype)
    s["v_rows"][:n] = _rows_at(s, v, vs, at).to(s["v_rows"].dtype)


def _attention(s, layer, out):
    """Every request over its own table, shared pages or not."""
    hd, nq, nkv, page, n = s["head_dim"], s["q_heads"], s["kv_heads"], s["page"], s["total"]
    cu, start = s["cu"].long(), s["start"].long()
    n_req, cols, most = start.numel(), -(-s["longest"] // page), s["most_rows"]
    keys = torch.arange(cols * page, device=cu.device)
    pages = s["table"][:, :cols].long().clamp(min=0)

    def gathered(x, scale):
        x = x[pages].float() if scale is None else _values(x.view(torch.uint8)[pages], scale[pages])
        return x.transpose(1, 2).reshape(n_req, nkv, cols * page, hd)

    k, v = gathered(*layer[:2]), gathered(*layer[2:])
    # a request's rows, padded to the most that one brings
    i = torch.arange(most, device=cu.device)
    row = (cu[:-1, None] + i).clamp(max=s["room"] - 1)
    pos = (start[:, None] + i).clamp(max=s["rope"].shape[0] - 1)
    q = s["qkv"][row][..., :nq * hd].view(n_req, most, nq, hd)
    q = _norm_rotate(q, s["gain"], s["rope"], pos).view(n_req, most, nkv, nq // nkv, hd).transpose(1, 2).reshape(n_req, nkv, -1, hd)
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(hd)
    hidden = keys > pos.repeat_interleave(nq // nkv, 1)[:, None, :, None]
    score.masked_fill_(hidden, -math.inf)
    p = (score - score.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
    o = o.view(n_req, nkv, most, nq // nkv, hd).transpose(1, 2).reshape(n_req, most, nq, hd)
    live = torch.arange(n, device=cu.device)
    req = torch.searchsorted(cu[1:], live, right=True)
    out[:n] = o[req, live - cu[req]].to(out.dtype)
    return out


def run(s):
    if own:
        _own(s)
    elif s["op"] in ("append", "read"):
        if s["op"] == "append":
            _append(s)
        _read(s, s["total"] if s["op"] == "append" else s["places"].numel())
    else:
        [_attention(s, layer, out) for layer, out in zip(s["layers"], s["out"])]
    return [s["k_rows"], s["v_rows"]] if s["op"] in ("append", "read") else s["out"]


# ------------------------------------------------------------------------------------------------ 64 bits

def _nearest_code(x):
    """x float64 rounded to the nearest e4m3 value, ties to even: steps of 2^-9 up to 2^-6, then an eighth of the power of two below."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _stored(x):
    """What float64 rows become in the cache."""
    k = torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / E4M3_MAX)).clamp(min=LEAST_SCALE - 127)
    return _nearest_code(x * torch.exp2(-k)) * torch.exp2(k)


def exact(c, seed):
    """Request by request, in float64, from the definitions."""
    s = prepare(c, seed)
    w = _layout(c)
    start, rows = w["start"], w["rows"]
    hd, nq, nkv, page = c["head_dim"], c["q_heads"], c["kv_heads"], c["page"]
    half, n = hd // 2, s["total"]

    def wide(x, scale):
        return x.double() if scale is None else x.double() * torch.exp2(scale.double() - 127).unsqueeze(-1)

    if c["op"] == "read":
        at = s["places"]
        return [wide(x.view(torch.uint8)[at // page, :, at % page].view(torch.float8_e4m3fn) if c["dtype"] == "e4m3" else x[at // page, :, at % page],
                     None if scale is None else scale[at // page, :, at % page]) for x, scale in (s["layers"][0][:2], s["layers"][0][2:])]
    x = s["qkv"].double().view(-1, nq + 2 * nkv, hd)
    heads = x[:n, :nq + nkv]
    heads = heads * s["gain"].double() / (heads.pow(2).sum(-1, keepdim=True) / hd + EPS).sqrt()
    angles = s["rope"][s["pos"][:n].long()].double()
    cos, sin = angles[:, None, :, 0], angles[:, None, :, 1]
    turned = torch.empty_like(heads)
    turned[..., :half] = heads[..., :half] * cos - heads[..., half:] * sin
    turned[..., half:] = heads[..., half:] * cos + heads[..., :half] * sin
    if c["op"] == "append":
        k, v = torch.zeros(s["room"], nkv, hd, device="cuda", dtype=torch.float64), torch.zeros(s["room"], nkv, hd, device="cuda", dtype=torch.float64)
        k[:n], v[:n] = _stored(turned[:, nq:]), _stored(x[:n, nq + nkv:])
        return [k, v]
    outs = []
    for layer in s["layers"]:
        out, at = torch.zeros(s["room"], nq, hd, device="cuda", dtype=torch.float64), 0
        for i, (first, count) in enumerate(zip(start, rows)):
            if not count:
                continue
            where = torch.arange(first, first + count, device="cuda")
            seen = torch.arange(first + count, device="cuda") <= where[:, None]
            pages = s["table"][i, :-(-(first + count) // page)].long()
            for g in range(nkv):
                k, v = (wide(x[:, g].view(torch.uint8)[pages].view(torch.float8_e4m3fn) if c["dtype"] == "e4m3" else x[:, g][pages],
                             None if scale is None else scale[pages, g]).reshape(-1, hd)[:first + count] for x, scale in (layer[:2], layer[2:]))
                q = turned[at:at + count, g * (nq // nkv):(g + 1) * (nq // nkv)].transpose(0, 1)
                z = torch.matmul(q, k.T) * hd ** -0.5
                out[at:at + count, g * (nq // nkv):(g + 1) * (nq // nkv)] = torch.matmul(torch.softmax(z.masked_fill(~seen, -math.inf), -1), v).transpose(0, 1)
            at += count
        outs.append(out)
    return outs
