"""Workloads of the paged key-value cache's operators (append, attend, evict) and their plain forms.

A serving process holds, per layer, a pool of pages; every active request owns some of them through a table.  One
decode slot appends one token per request and attends over all of its tokens; a prompt is appended at once; eviction
keeps the tokens that attention has used most.  Capacities (4 096 .. 262 144 tokens), active sets (up to 512
requests), request lengths (up to 16 384 tokens) and the 2 048 prompt tokens a slot may load are those of the
simulator's presets; head counts and widths are common ones.

``own = False``: elementary torch operations in 32 bits.  ``own = True``: the library's calls.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
SIZES = {"bf16": 2, "f16": 2, "e4m3": 1}
EPS = 1e-6


def _append(name, requests, each, heads, kv_heads, head_dim, dtype, cache, rope_dim, page, **kw):
    return dict(name=name, op="append", requests=requests, each=each, heads=heads, kv_heads=kv_heads,
                head_dim=head_dim, dtype=dtype, cache=cache, rope_dim=rope_dim, page=page,
                interleaved=kw.get("interleaved", False), norm=kw.get("norm", True),
                heads_first=kw.get("heads_first", False), longest=kw.get("longest", 8192))


def _attend(name, requests, law, longest, heads, kv_heads, head_dim, dtype, cache, page, **kw):
    return dict(name=name, op="attend", requests=requests, law=law, longest=longest, heads=heads, kv_heads=kv_heads,
                head_dim=head_dim, dtype=dtype, cache=cache, page=page, weight=kw.get("weight", False),
                window=kw.get("window", 0), heads_first=kw.get("heads_first", False))


def _evict(name, requests, law, longest, budget, recent, first, kv_heads, head_dim, cache, page, **kw):
    return dict(name=name, op="evict", requests=requests, law=law, longest=longest, budget=budget, recent=recent,
                first=first, kv_heads=kv_heads, head_dim=head_dim, cache=cache, page=page,
                heads_first=kw.get("heads_first", False))


def listed():
    return [
        # one request decoding alone: the smallest call there is, latency only
        _append("append one token", 1, 1, 32, 8, 128, "bf16", "bf16", 128, 16),
        # a decode slot of a full active set (256 requests), half-rotated heads, f16
        _append("append a slot f16", 256, 1, 64, 8, 128, "f16", "f16", 64, 16, interleaved=True, heads_first=True),
        # the most prompt tokens a slot may load (2 048), in two prompts, stored in 8 bits; an odd head width
        _append("append prompts e4m3", 2, 1024, 48, 6, 96, "bf16", "e4m3", 96, 48),
        # the longest prompts at once
        _append("append long prompts", 2, 8192, 64, 8, 128, "bf16", "bf16", 128, 64),
        # one short request: latency only
        _attend("attend one short", 1, "even", 129, 32, 8, 128, "bf16", "bf16", 16),
        # one request that owns the whole cache of 131 072 tokens: split over the length
        _attend("attend one long", 1, "even", 131072, 32, 8, 128, "bf16", "bf16", 16),
        # 100 requests of lognormal prompts, small f16 heads, with the weights that eviction needs
        _attend("attend ragged f16 weight", 100, "lognormal", 4096, 25, 5, 64, "f16", "f16", 16, weight=True),
        # a cache of 131 072 tokens in 8 bits, heads outermost, a window of 4 096
        _attend("attend e4m3", 64, "lognormal", 16384, 64, 8, 128, "bf16", "e4m3", 64, window=4096,
                heads_first=True),
        # a heavy-tailed active set that fills a cache of about 262 144 tokens
        _attend("attend heavy tailed", 128, "heavy", 16384, 64, 8, 128, "bf16", "bf16", 16),
        # a few short requests cut to half
        _evict("evict few", 4, "even", 515, 256, 32, 4, 8, 64, "bf16", 16),
        # an active set cut to 1 024 tokens a request
        _evict("evict active set", 64, "lognormal", 4096, 1024, 128, 4, 8, 128, "bf16", 16),
        # long requests cut to an eighth, 8 bits, heads outermost
        _evict("evict long e4m3", 4, "even", 65536, 8192, 512, 16, 8, 128, "e4m3", 64, heads_first=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("append", "attend", "attend", "evict"))
    dtype = rng.choice(("bf16", "f16"))
    cache = rng.choice((dtype, dtype, "e4m3"))
    head_dim = rng.choice((64, 80, 96, 112, 128, 128, 192, 256))
    kv_heads = rng.choice((1, 2, 4, 5, 8))
    group = rng.choice((1, 2, 3, 4, 5, 7, 8, 8, 12, 16))
    heads = kv_heads * group
    page = rng.choice((8, 16, 16, 24, 32, 64, 128))
    first = rng.random() < 0.5
    if op == "append":
        room = 16384 * 80 * 128 // ((heads + 2 * kv_heads) * head_dim)
        if rng.random() < 0.5:
            requests, each = _log(rng, 1, 512), 1
        else:
            requests = rng.randint(1, 4)
            each = _log(rng, 2, min(8192, room) // requests)
        rope_dim = rng.choice((head_dim, 64))
        c = _append("", requests, each, heads, kv_heads, head_dim, dtype, cache, rope_dim, page,
                    interleaved=rng.random() < 0.3, norm=rng.random() < 0.8, heads_first=first)
    elif op == "attend":
        law = rng.choice(("even", "lognormal", "heavy"))
        requests = _log(rng, 1, 512)
        # padded tokens of the plain form, and tokens of the cache, within the largest listed case
        tokens = 262144 * 8 * 128 // (kv_heads * head_dim)
        longest = _log(rng, 1, max(2, min(131072 if requests == 1 else 16384, tokens * 2 // requests)))
        if law == "even":
            longest = min(longest, max(1, tokens // requests))
        weight = rng.random() < 0.4
        window = rng.choice((0, 0, 0, _log(rng, 1, longest)))
        c = _attend("", requests, law, longest, heads, kv_heads, head_dim, dtype, cache, page, weight=weight,
                    window=window, heads_first=first)
    else:
        requests = _log(rng, 1, 64)
        tokens = 262144 * 8 * 128 // (kv_heads * head_dim)
        longest = _log(rng, 64, min(65536, tokens // requests))
        budget = _log(rng, max(1, longest // 16), max(2, longest * 3 // 4))
        budget = min(budget, max(1, tokens // 4 // requests))
        c = _evict("", requests, rng.choice(("even", "lognormal", "heavy")), longest, budget,
                   rng.randint(0, budget // 4), rng.randint(0, min(8, budget // 4)), kv_heads, head_dim, cache, page,
                   heads_first=first)
    del c["name"]
    return c


def _lengths(case):
    """The lengths of a case's requests: a property of the case (their order goes by the seed)."""
    n, top = case["requests"], case["longest"]
    rng = random.Random(n * 1000003 + top)
    if case["law"] == "even":  # all within a page of the longest
        got = [max(1, top - rng.randint(0, 16)) if i else top for i in range(n)]
    elif case["law"] == "lognormal":  # lognormal prompts and geometric output
        got = [int(rng.lognormvariate(math.log(max(2, top) / 6), 1.0)) + int(rng.expovariate(1 / (1 + top / 20)))
               for _ in range(n)]
    else:  # 70 % short prompts, 30 % long ones, and a Pareto output
        got = [(rng.randint(max(1, top // 512), max(1, top // 64)) if rng.random() < 0.7 else
                rng.randint(max(1, top // 8), max(1, top // 2))) + int(16 * rng.paretovariate(1.5)) for _ in range(n)]
    return [max(1, min(top, x)) for x in got]


def _pool(g, pages, page, kv_heads, head_dim, cache, heads_first):
    """[pages, page, kv_heads, head_dim], of either memory order; values as normalised keys have them."""
    shape = (pages, kv_heads, page, head_dim) if heads_first else (pages, page, kv_heads, head_dim)
    x = torch.randn(shape, device="cuda", generator=g, dtype=torch.float16).to(DTYPES[cache])
    return x.transpose(1, 2) if heads_first else x


def _tables(order, lengths, page, width=None, at=0):
    """Pages for requests of the given lengths, taken from `order` from place `at` on; unused entries are -1."""
    need = (lengths + page - 1) // page
    width = int(need.max()) if width is None else width
    cols = torch.arange(width, device=order.device)
    start = torch.cumsum(need, 0) - need + at
    used = cols[None, :] < need[:, None]
    place = (start[:, None] + cols[None, :]).clamp(max=order.numel() - 1)
    return torch.where(used, order[place], torch.full_like(place, -1)).to(torch.int32), int(need.sum())


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 17)
    page, kv_heads, head_dim = case["page"], case["kv_heads"], case["head_dim"]
    s = {"case": case}

    def randn(*shape, dtype=torch.float32):
        return torch.randn(shape, device="cuda", generator=g).to(dtype)

    def scales():
        if case["cache"] != "e4m3":
            return None
        return 0.25 + 0.5 * torch.rand(kv_heads, device="cuda", generator=g)

    if case["op"] == "append":
        n, each, dtype = case["requests"] * case["each"], case["each"], DTYPES[case["dtype"]]
        held = torch.randint(1, case["longest"], (case["requests"],), device="cuda", generator=g)
        if each > 1:
            held = torch.zeros_like(held)  # prompts start at position 0
        per = (each + page - 1) // page + 1
        pages = case["requests"] * per + 7
        order = torch.randperm(pages, device="cuda", generator=g)[:case["requests"] * per].view(case["requests"], per)
        pos = held[:, None] + torch.arange(each, device="cuda")[None, :]
        inside = pos - (held // page * page)[:, None]
        s["positions"] = pos.reshape(-1).to(torch.int32)
        s["slots"] = (torch.gather(order, 1, inside // page) * page + inside % page).reshape(-1).to(torch.int64)
        # q, k and v come as one projection's output
        x = randn(n, (case["heads"] + 2 * kv_heads) * head_dim, dtype=dtype)
        h = case["heads"] * head_dim
        w = kv_heads * head_dim
        s["q"] = x[:, :h].view(n, case["heads"], head_dim)
        s["k"] = x[:, h:h + w].view(n, kv_heads, head_dim)
        s["v"] = x[:, h + w:].view(n, kv_heads, head_dim)
        s["q_norm"] = (1 + 0.1 * randn(head_dim)).to(dtype) if case["norm"] else None
        s["k_norm"] = (1 + 0.1 * randn(head_dim)).to(dtype) if case["norm"] else None
        r = case["rope_dim"]
        freq = 10000.0 ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r)
        angle = torch.arange(case["longest"] + each, device="cuda", dtype=torch.float64)[:, None] * freq[None, :]
        s["rope"] = torch.cat((angle.cos(), angle.sin()), 1).float()
        weight = torch.rand(pages, kv_heads, page, device="cuda", generator=g)
    else:
        lengths = torch.tensor(_lengths(case), device="cuda", dtype=torch.int64)
        lengths = lengths[torch.randperm(lengths.numel(), device="cuda", generator=g)]
        live = int(((lengths + page - 1) // page).sum())
        spare = case["requests"] * (-(-case["budget"] // page)) if case["op"] == "evict" else 0
        pages = live + spare + 7
        order = torch.randperm(pages, device="cuda", generator=g)
        s["table"], used = _tables(order, lengths, page)
        s["lengths"] = lengths.to(torch.int32)
        weight = torch.exp(2 * randn(pages, kv_heads, page))
        if case["op"] == "evict":
            weight = weight * (torch.rand(weight.shape, device="cuda", generator=g) > 0.02)  # new tokens have none
            s["budget"] = torch.full_like(s["lengths"], case["budget"])
            s["new_table"], _ = _tables(order, s["budget"].long(), page, at=used)
    s["k_cache"] = _pool(g, pages, page, kv_heads, head_dim, case["cache"], case["heads_first"])
    s["v_cache"] = _pool(g, pages, page, kv_heads, head_dim, case["cache"], case["heads_first"])
    s["k_scale"], s["v_scale"] = scales(), scales()
    s["weight"] = weight.contiguous()
    if case["op"] == "attend":
        s["q"] = randn(case["requests"], case["heads"], head_dim, dtype=DTYPES[case["dtype"]])
        # some tokens of each request are what its queries look for (the same key, so that a token may be drawn twice)
        b = torch.arange(case["requests"], device="cuda").repeat_interleave(4)
        t = (torch.rand(b.numel(), device="cuda", generator=g) * lengths[b]).long()
        at = s["table"].long()[b, t // page]
        look = s["q"].float().view(case["requests"], kv_heads, -1, head_dim).mean(2)[b]
        near = 2 * look + randn(case["requests"], kv_heads, head_dim)[b]
        _put(s["k_cache"], at, t % page, near)
    if own:  # what a serving process keeps for as long as its pages: the object that names them
        from paper_2604_11001_b200.kvcache import PagedKV
        s["cache"] = PagedKV(s["k_cache"], s["v_cache"], weight=s["weight"], k_scale=s["k_scale"],
                             v_scale=s["v_scale"])
    return s


# ------------------------------------------------------------------------------------------------- plain forms
def _rows(cache, pages, places):
    """Rows of the pool in 32 bits: [..., kv_heads, head_dim] for index tensors of one shape."""
    if cache.dtype == torch.float8_e4m3fn:
        return cache.view(torch.uint8)[pages, places].view(torch.float8_e4m3fn).float()
    return cache[pages, places].float()


def _put(cache, pages, places, rows):
    if cache.dtype == torch.float8_e4m3fn:
        cache.view(torch.uint8)[pages, places] = rows.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        cache[pages, places] = rows.to(cache.dtype)


def _normed(x, w):
    x = x.float()
    if w is None:
        return x
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()


def _rotated(x, rope, positions, r, interleaved):
    cs = rope[positions.long()][:, None, :]
    cos, sin = cs[..., :r // 2], cs[..., r // 2:]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., r:]), -1)


def _plain_append(s):
    c = s["case"]
    page = c["page"]
    q = _rotated(_normed(s["q"], s["q_norm"]), s["rope"], s["positions"], c["rope_dim"], c["interleaved"])
    k = _rotated(_normed(s["k"], s["k_norm"]), s["rope"], s["positions"], c["rope_dim"], c["interleaved"])
    v = s["v"].float()
    if s["k_scale"] is not None:
        k = k / s["k_scale"][None, :, None]
        v = v / s["v_scale"][None, :, None]
    at, place = s["slots"] // page, s["slots"] % page
    _put(s["k_cache"], at, place, k)
    _put(s["v_cache"], at, place, v)
    s["weight"].transpose(1, 2)[at, place] = 0
    return q.to(s["q"].dtype), s["k_cache"], s["v_cache"], s["weight"]


def _live(s):
    """The pages and places of all tokens of all requests, padded to the longest."""
    page = s["case"]["page"]
    t = torch.arange(s["table"].shape[1] * page, device="cuda")
    pages = s["table"].long().clamp(min=0)[:, t // page]
    return t, pages, (t % page).expand_as(pages)


def _plain_attend(s):
    c = s["case"]
    B, Hk, D = c["requests"], c["kv_heads"], c["head_dim"]
    t, pages, places = _live(s)
    k, v = _rows(s["k_cache"], pages, places), _rows(s["v_cache"], pages, places)
    q = s["q"].float().view(B, Hk, -1, D) * (D ** -0.5)
    if s["k_scale"] is not None:
        q = q * s["k_scale"][None, :, None, None]
    logits = torch.matmul(q, k.permute(0, 2, 3, 1))
    n = s["lengths"].long()[:, None]
    live = t[None, :] < n
    if c["window"]:
        live = live & (t[None, :] >= n - c["window"])
    logits = logits.masked_fill(~live[:, None, None, :], float("-inf"))
    top = logits.amax(-1, keepdim=True)
    e = torch.exp(logits - top)
    total = e.sum(-1, keepdim=True)
    p = e / total
    out = torch.matmul(p, v.transpose(1, 2))
    if s["v_scale"] is not None:
        out = out * s["v_scale"][None, :, None, None]
    lse = (torch.log(total) + top).view(B, -1)
    out = out.reshape(B, -1, D).to(s["q"].dtype)
    if not c["weight"]:
        return out, lse
    more = p.sum(2)  # [B, Hk, t]
    b, at = live.nonzero(as_tuple=True)
    w = s["weight"].transpose(1, 2)
    pg, pl = pages[b, at], places[b, at]
    w[pg, pl] = w[pg, pl] + more.transpose(1, 2)[b, at]
    return out, lse, s["weight"]


def _plain_evict(s):
    c = s["case"]
    page, B, Hk, top = c["page"], c["requests"], c["kv_heads"], c["budget"]
    t, pages, places = _live(s)
    n, budget = s["lengths"].long()[:, None], s["budget"].long()[:, None]
    recent = budget.clamp(max=c["recent"])
    first = (budget - recent).clamp(max=c["first"])
    w = s["weight"].transpose(1, 2)[pages, places].transpose(1, 2)  # [B, Hk, t]
    live = t[None, :] < n
    sure = live & ((t[None, :] < first) | (t[None, :] >= n - recent))
    key = w.masked_fill(sure[:, None, :], float("inf")).masked_fill(~live[:, None, :], float("-inf"))
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices
    new = torch.minimum(n, budget)  # [B, 1]
    chosen = torch.zeros_like(key, dtype=torch.bool)
    chosen.scatter_(2, order, (t[None, :] < new)[:, None, :].expand_as(order))
    b, h, at = chosen.nonzero(as_tuple=True)
    to = (torch.cumsum(chosen, -1) - 1)[b, h, at]
    kept = torch.full((B, Hk, top), -1, dtype=torch.int32, device="cuda")
    kept[b, h, to] = at.to(torch.int32)
    new_page, new_place = s["new_table"].long()[b, to // page], to % page
    old_page, old_place = pages[b, at], at % page
    byte = torch.uint8 if c["cache"] == "e4m3" else torch.int16
    for pool in (s["k_cache"].view(byte), s["v_cache"].view(byte)):
        pool[new_page, new_place, h] = pool[old_page, old_place, h]
    s["weight"][new_page, h, new_place] = s["weight"][old_page, h, old_place]
    return new[:, 0].to(torch.int32), kept, s["k_cache"], s["v_cache"], s["weight"]


def run(s):
    c = s["case"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "evict": _plain_evict}[c["op"]](s)
    cache = s["cache"]
    if c["op"] == "append":
        q = cache.append(s["q"], s["k"], s["v"], s["positions"], s["slots"], rope=s["rope"],
                         interleaved=c["interleaved"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS)
        return q, cache.k, cache.v, cache.weight
    if c["op"] == "attend":
        out, lse = cache.attend(s["q"], s["table"], s["lengths"], window=c["window"], add_weight=c["weight"],
                                return_lse=True)
        return (out, lse, cache.weight) if c["weight"] else (out, lse)
    new, kept = cache.evict(s["table"], s["lengths"], s["budget"], s["new_table"], max_budget=c["budget"],
                            recent=c["recent"], first=c["first"])
    return new, kept, cache.k, cache.v, cache.weight


# ------------------------------------------------------------------------------------------------- what it takes
def work(case):
    Hk, D, size = case["kv_heads"], case["head_dim"], SIZES[case["cache"]]
    if case["op"] == "append":
        n = case["requests"] * case["each"]
        rows = n * (case["heads"] * 2 * 2 + Hk * 2 * (2 + size)) * D
        angles = min(n, case["longest"] + case["each"]) * case["rope_dim"] * 4
        return {"bytes": rows + angles + n * (4 + 8 + 4 * Hk),
                "flops": n * (case["heads"] + Hk) * (4 * D + 3 * case["rope_dim"])}
    lengths = _lengths(case)
    if case["op"] == "attend":
        seen = sum(min(x, case["window"]) if case["window"] else x for x in lengths)
        more = seen * Hk * 8 if case["weight"] else 0
        ends = case["requests"] * case["heads"] * (4 * D + 4)
        return {"bytes": seen * Hk * D * 2 * size + ends + more + 4 * (seen // case["page"] + case["requests"]),
                "flops": 4 * seen * case["heads"] * D}
    kept = sum(min(x, case["budget"]) for x in lengths) * Hk
    return {"bytes": sum(lengths) * Hk * 4 + kept * (2 * 2 * D * size + 4 + 4), "flops": sum(lengths) * Hk}


# ------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    page, Hk, D = case["page"], case["kv_heads"], case["head_dim"]
    wide = torch.float64

    def row(cache, pages, places):
        x = cache.view(torch.uint8)[pages, places].view(torch.float8_e4m3fn) if case["cache"] == "e4m3" else cache[pages, places]
        return x.to(wide)

    if case["op"] == "append":
        r, half = case["rope_dim"], case["rope_dim"] // 2
        at = torch.arange(r, device="cuda")
        mate = (at ^ 1) if case["interleaved"] else (at + half) % r
        which = at // 2 if case["interleaved"] else at % half
        sign = torch.where((at % 2 if case["interleaved"] else at // half) == 0, -1.0, 1.0).to(wide)
        angle = s["rope"].to(wide)[s["positions"].long()]
        cos, sin = angle[:, which][:, None], (angle[:, half + which] * sign)[:, None]
        out = []
        for x, w in ((s["q"], s["q_norm"]), (s["k"], s["k_norm"])):
            x = x.to(wide)
            if w is not None:
                x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / D + EPS) * w.to(wide)
            x[..., :r] = x[..., :r] * cos + x[..., :r][..., mate] * sin
            out.append(x)
        out.append(s["v"].to(wide))
        pools = []
        for x, name in ((out[1], "k"), (out[2], "v")):
            pool = s[name + "_cache"].to(wide)
            if case["cache"] == "e4m3":
                x = (x / s[name + "_scale"].to(wide)[:, None]).clamp(-448, 448)
            pool[s["slots"] // page, s["slots"] % page] = x
            pools.append(pool)
        weight = s["weight"].to(wide)
        weight[s["slots"] // page, :, s["slots"] % page] = 0
        return out[0], pools[0], pools[1], weight
    lengths = s["lengths"].tolist()
    if case["op"] == "attend":
        outs, lses, weight = [], [], s["weight"].to(wide)
        for b, n in enumerate(lengths):
            t = torch.arange(max(0, n - case["window"]) if case["window"] else 0, n, device="cuda")
            pages, places = s["table"][b].long()[t // page], t % page
            k, v = row(s["k_cache"], pages, places), row(s["v_cache"], pages, places)
            if case["cache"] == "e4m3":
                k, v = k * s["k_scale"].to(wide)[:, None], v * s["v_scale"].to(wide)[:, None]
            q = s["q"][b].to(wide).view(Hk, -1, D)
            logits = torch.bmm(q, k.permute(1, 2, 0)) / math.sqrt(D)
            lse = torch.logsumexp(logits, -1)
            p = torch.exp(logits - lse[..., None])
            outs.append(torch.bmm(p, v.transpose(0, 1)).reshape(-1, D))
            lses.append(lse.reshape(-1))
            if case["weight"]:
                weight[pages, :, places] += p.sum(1).T
        return (torch.stack(outs), torch.stack(lses)) + ((weight,) if case["weight"] else ())
    if sum(lengths) * Hk > 1 << 23:  # selection on the host: minutes beyond this
        return None
    weight, k, v = s["weight"].to(wide), s["k_cache"].to(wide), s["v_cache"].to(wide)
    kept = torch.full((case["requests"], Hk, case["budget"]), -1, dtype=torch.int32)
    new_lengths = []
    for b, n in enumerate(lengths):
        keep = min(n, case["budget"])
        recent = min(case["recent"], case["budget"])
        first = min(case["first"], case["budget"] - recent)
        t = torch.arange(n, device="cuda")
        pages, places = s["table"][b].long()[t // page], t % page
        w = weight[pages, :, places].cpu().numpy()
        new_lengths.append(keep)
        for h in range(Hk):
            mine = w[:, h].tolist()
            order = sorted(range(n), key=lambda i: (0 if i < first or i >= n - recent else 1, -mine[i], i))
            kept[b, h, :keep] = torch.tensor(sorted(order[:keep]), dtype=torch.int32)
            at = kept[b, h, :keep].long().cuda()
            to = torch.arange(keep, device="cuda")
            np_, nl = s["new_table"][b].long()[to // page], to % page
            k[np_, nl, h], v[np_, nl, h] = k[pages[at], places[at], h], v[pages[at], places[at], h]
            weight[np_, h, nl] = weight[pages[at], h, places[at]]
    return torch.tensor(new_lengths, dtype=torch.int32), kept, k, v, weight
