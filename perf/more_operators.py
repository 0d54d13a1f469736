"""Workloads of the paged key-value cache's prompt attention (prefill), of attention over a window and the first tokens
(attend with `first`) and of reading the cache back (read), and their plain forms.

A serving process loads prompts whole or in chunks (the simulator's presets: at most 2 048 prompt tokens a slot, chunks of
512) and then attends with one token per request and slot.  Models with a sliding window keep a few first tokens visible.
Capacities (4 096 .. 131 072 tokens), active sets (up to 256 requests) and request lengths (up to 16 384 tokens) are those
of the simulator's presets; head counts and widths are common ones.

``own = False``: elementary torch operations in 32 bits.  ``own = True``: the library's calls.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
SIZES = {"bf16": 2, "f16": 2, "e4m3": 1}
PAIRS = 8192 * 8192 * 32     # (row, head, key) triples of the plain form's padded logits, at most
TOKENS = 262144              # padded tokens of 8 heads of 128 that the plain form holds in 32 bits, at most


def _prefill(name, requests, law, new, context, heads, kv_heads, head_dim, dtype, cache, page, **kw):
    return dict(name=name, op="prefill", requests=requests, law=law, new=new, context=context, heads=heads,
                kv_heads=kv_heads, head_dim=head_dim, dtype=dtype, cache=cache, page=page, window=kw.get("window", 0),
                first=kw.get("first", 0), heads_first=kw.get("heads_first", False))


def _attend(name, requests, law, longest, heads, kv_heads, head_dim, dtype, cache, page, window, first, **kw):
    return dict(name=name, op="attend", requests=requests, law=law, longest=longest, heads=heads, kv_heads=kv_heads,
                head_dim=head_dim, dtype=dtype, cache=cache, page=page, window=window, first=first,
                weight=kw.get("weight", False), heads_first=kw.get("heads_first", False))


def _read(name, requests, law, longest, kv_heads, head_dim, cache, to, page, **kw):
    return dict(name=name, op="read", requests=requests, law=law, longest=longest, kv_heads=kv_heads,
                head_dim=head_dim, cache=cache, to=to, page=page, heads_first=kw.get("heads_first", False))


def listed():
    return [
        # one short prompt: the smallest call there is, latency only
        _prefill("prefill one short", 1, "even", 64, 0, 32, 8, 128, "bf16", "bf16", 16),
        # the most prompt tokens a slot may load (2 048), in twelve prompts of uneven length
        _prefill("prefill a slot", 12, "lognormal", 512, 0, 64, 8, 128, "bf16", "bf16", 16),
        # chunks of 512 behind long contexts, a window of 4 096 and four first tokens
        _prefill("prefill chunks window f16", 4, "even", 512, 16384, 32, 8, 128, "f16", "f16", 64, window=4096, first=4,
                 heads_first=True),
        # the last few tokens of long prompts, over 8 bits: bound by the cache's bytes
        _prefill("prefill few tokens e4m3", 16, "lognormal", 7, 16384, 64, 8, 128, "bf16", "e4m3", 64),
        # odd widths, groups and pages, a short window
        _prefill("prefill odd f16", 6, "lognormal", 700, 300, 25, 5, 80, "f16", "f16", 24, window=200, first=3),
        # a long prompt at once
        _prefill("prefill long prompt", 1, "even", 8192, 0, 32, 8, 128, "bf16", "bf16", 16),
        # one long request, of which a window and four first tokens are seen
        _attend("attend one first", 1, "even", 131072, 32, 8, 128, "bf16", "bf16", 16, 4096, 4),
        # an active set: a window of 1 024 and sixteen first tokens
        _attend("attend slot first", 128, "lognormal", 8192, 64, 8, 128, "bf16", "bf16", 16, 1024, 16),
        # in 8 bits, with the weights that eviction needs, heads outermost
        _attend("attend first e4m3 weight", 64, "lognormal", 16384, 64, 8, 128, "bf16", "e4m3", 64, 2048, 64, weight=True,
                heads_first=True),
        # a page of one request
        _read("read one page", 1, "even", 16, 8, 128, "bf16", "bf16", 16),
        # uneven requests out of 8 bits, odd widths
        _read("read ragged e4m3", 32, "lognormal", 2048, 5, 80, "e4m3", "f16", 24),
        # long requests out of 8 bits, as they are moved to another cache
        _read("read long e4m3", 4, "even", 32768, 8, 128, "e4m3", "bf16", 64, heads_first=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("prefill", "prefill", "attend", "read"))
    dtype = rng.choice(("bf16", "f16"))
    cache = rng.choice((dtype, dtype, "e4m3"))
    head_dim = rng.choice((64, 80, 96, 112, 128, 128, 192, 256))
    kv_heads = rng.choice((1, 2, 4, 5, 8))
    heads = kv_heads * rng.choice((1, 2, 3, 4, 5, 7, 8, 8, 12, 16))
    page = rng.choice((8, 16, 16, 24, 32, 64, 128))
    law = rng.choice(("even", "lognormal"))
    first = rng.random() < 0.5
    tokens = TOKENS * 8 * 128 // (kv_heads * head_dim)
    if op == "prefill":
        requests = _log(rng, 1, 32)
        new = _log(rng, 1, 4096 if requests <= 4 else 1024)
        room = min(tokens // requests, 16384, PAIRS // (requests * new * heads))
        new = max(1, min(new, room // 2))
        context = 0 if rng.random() < 0.4 else _log(rng, 1, max(2, room - new))
        window = rng.choice((0, 0, _log(rng, 1, max(2, new + context))))
        c = _prefill("", requests, law, new, context, heads, kv_heads, head_dim, dtype, cache, page, window=window,
                     first=rng.randint(0, 70) if window else 0, heads_first=first)
    elif op == "attend":
        requests = _log(rng, 1, 256)
        longest = _log(rng, 16, max(17, min(131072 if requests == 1 else 16384, tokens * 2 // requests)))
        if law == "even":
            longest = min(longest, max(16, tokens // requests))
        c = _attend("", requests, law, longest, heads, kv_heads, head_dim, dtype, cache, page, _log(rng, 1, longest),
                    rng.randint(1, 70), weight=rng.random() < 0.4, heads_first=first)
    else:
        requests = _log(rng, 1, 64)
        longest = _log(rng, 1, max(2, min(32768, tokens // 2 // requests)))
        c = _read("", requests, law, longest, kv_heads, head_dim, cache,
                  dtype if cache != "e4m3" else rng.choice(("bf16", "f16")), page, heads_first=first)
    del c["name"]
    return c


def _lengths(case):
    """The requests' new tokens and lengths: a property of the case (their order goes by the seed)."""
    n = case["requests"]
    rng = random.Random(n * 1000003 + case.get("new", 0) * 7 + case.get("context", case.get("longest")))

    def some(top):
        if case["law"] == "even":  # all within a page of the longest
            return [max(1, top - rng.randint(0, 16)) if i else top for i in range(n)]
        return [max(1, min(top, int(rng.lognormvariate(math.log(max(2, top) / 4), 1.0)))) for _ in range(n)]
    if case["op"] != "prefill":
        x = some(case["longest"])
        return x, x
    new = some(case["new"])
    before = some(case["context"]) if case["context"] else [0] * n
    return new, [a + b for a, b in zip(new, before)]


def _pool(g, pages, page, kv_heads, head_dim, cache, heads_first):
    """[pages, page, kv_heads, head_dim], of either memory order; values as normalised keys have them."""
    shape = (pages, kv_heads, page, head_dim) if heads_first else (pages, page, kv_heads, head_dim)
    x = torch.randn(shape, device="cuda", generator=g, dtype=torch.float16).to(DTYPES[cache])
    return x.transpose(1, 2) if heads_first else x


def _bytes(pool):
    """A view that can be indexed."""
    return pool.view(torch.uint8) if pool.dtype == torch.float8_e4m3fn else pool


def _rows(pool, pages, places, as_type=torch.float32):
    x = _bytes(pool)[pages, places]
    return (x.view(torch.float8_e4m3fn) if pool.dtype == torch.float8_e4m3fn else x).to(as_type)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 29)
    page, kv_heads, head_dim, requests = case["page"], case["kv_heads"], case["head_dim"], case["requests"]

    def randn(*shape, dtype=torch.float32):
        return torch.randn(shape, device="cuda", generator=g).to(dtype)

    order = torch.randperm(requests, device="cuda", generator=g)
    new, lengths = (torch.tensor(x, device="cuda", dtype=torch.int64)[order] for x in _lengths(case))
    need = (lengths + page - 1) // page
    pages = int(need.sum()) + 7
    taken = torch.randperm(pages, device="cuda", generator=g)
    cols = torch.arange(int(need.max()), device="cuda")
    place = (torch.cumsum(need, 0) - need)[:, None] + cols[None, :]
    table = torch.where(cols[None, :] < need[:, None], taken[place.clamp(max=pages - 1)], torch.full_like(place, -1))
    s = {"case": case, "table": table.to(torch.int32), "lengths": lengths.to(torch.int32)}
    for name in ("k", "v"):
        s[name + "_cache"] = _pool(g, pages, page, kv_heads, head_dim, case["cache"], case["heads_first"])
        s[name + "_scale"] = 0.25 + 0.5 * torch.rand(kv_heads, device="cuda", generator=g) if case["cache"] == "e4m3" else None
    s["weight"] = None
    starts = torch.cat((torch.zeros_like(new[:1]), torch.cumsum(new, 0)))
    rows = int(starts[-1])
    if case["op"] == "read":
        request = torch.repeat_interleave(torch.arange(requests, device="cuda"), new)
        token = torch.arange(rows, device="cuda") - starts[request]
        s["slots"] = table[request, token // page] * page + token % page
    else:
        n = rows if case["op"] == "prefill" else requests
        # q comes as a part of one projection's output
        x = randn(n, (case["heads"] + 2 * kv_heads) * head_dim, dtype=DTYPES[case["dtype"]])
        s["q"] = x[:, :case["heads"] * head_dim].view(n, case["heads"], head_dim)
        s["starts"] = starts.to(torch.int32)
        # some tokens of each request are what one of its queries looks for (the same key, so that a token may be drawn twice)
        b = torch.arange(requests, device="cuda").repeat_interleave(4)
        t = (torch.rand(b.numel(), device="cuda", generator=g) * lengths[b]).long()
        row = torch.rand(requests, device="cuda", generator=g)
        row = starts[:-1] + (row * new).long() if case["op"] == "prefill" else torch.arange(requests, device="cuda")
        near = (2 * s["q"][row].float().view(requests, kv_heads, -1, head_dim).mean(2) + randn(requests, kv_heads, head_dim))[b]
        _bytes(s["k_cache"])[table[b, t // page], t % page] = _bytes(near.to(s["k_cache"].dtype))
        if case.get("weight"):
            s["weight"] = torch.exp(2 * randn(pages, kv_heads, page)).contiguous()
    if own:  # what a serving process keeps for as long as its pages: the object that names them
        from paper_2604_11001_b200.kvcache import PagedKV
        s["cache"] = PagedKV(s["k_cache"], s["v_cache"], weight=s["weight"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    return s


# ------------------------------------------------------------------------------------------------- plain forms
def _scaled(x, scale):
    return x if scale is None else x * scale.to(x.dtype)[:, None]


def _plain_read(s):
    page, to = s["case"]["page"], DTYPES[s["case"]["to"]]
    at, place = s["slots"] // page, s["slots"] % page
    return (_scaled(_rows(s["k_cache"], at, place), s["k_scale"]).to(to),
            _scaled(_rows(s["v_cache"], at, place), s["v_scale"]).to(to))


def _live(s):
    """The pages and places of all tokens of all requests, padded to the longest."""
    page = s["case"]["page"]
    t = torch.arange(int(s["table"].shape[1]) * page, device="cuda")
    return t, s["table"].long().clamp(min=0)[:, t // page], (t % page).expand(s["table"].shape[0], -1)


def _seen(c, t, position):
    """Which keys t a query at `position` sees."""
    seen = t <= position
    if c["window"]:
        seen = seen & ((t > position - c["window"]) | (t < c["first"]))
    return seen


def _softmax(logits, seen):
    """In the place of the logits: the weights; and the log-sum-exp.  What sees nothing has neither."""
    logits.masked_fill_(~seen, float("-inf"))
    top = logits.amax(-1, keepdim=True).clamp(min=-3e38)
    e = logits.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    e.div_(total.clamp(min=1e-37))
    return e, (torch.log(total) + top)[..., 0]


def _plain_prefill(s):
    c = s["case"]
    B, H, Hk, D = c["requests"], c["heads"], c["kv_heads"], c["head_dim"]
    t, pages, places = _live(s)
    k, v = _scaled(_rows(s["k_cache"], pages, places), s["k_scale"]), _scaled(_rows(s["v_cache"], pages, places), s["v_scale"])
    starts, lengths = s["starts"].long(), s["lengths"].long()
    new = starts[1:] - starts[:-1]
    i = torch.arange(c["new"], device="cuda")
    live = i[None, :] < new[:, None]
    row = (starts[:-1, None] + i[None, :]).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][row].float() * (D ** -0.5)                                  # [B, new, H, D]
    q = q.view(B, c["new"], Hk, H // Hk, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, -1, D)
    logits = torch.matmul(q, k.permute(0, 2, 3, 1)).view(B, Hk, H // Hk, c["new"], -1)
    position = (lengths - new)[:, None] + i[None, :]
    seen = _seen(c, t[None, None, :], position[:, :, None]) & live[:, :, None]
    p, lse = _softmax(logits, seen[:, None, None])
    out = torch.matmul(p.view(B, Hk, -1, p.shape[-1]), v.transpose(1, 2)).view(B, H, c["new"], D)
    return out.transpose(1, 2)[live].to(s["q"].dtype), lse.view(B, H, c["new"]).transpose(1, 2)[live]


def _plain_attend(s):
    c = s["case"]
    B, Hk, D = c["requests"], c["kv_heads"], c["head_dim"]
    t, pages, places = _live(s)
    k, v = _scaled(_rows(s["k_cache"], pages, places), s["k_scale"]), _scaled(_rows(s["v_cache"], pages, places), s["v_scale"])
    q = s["q"].float().view(B, Hk, -1, D) * (D ** -0.5)
    seen = _seen(c, t[None, :], s["lengths"].long()[:, None] - 1)
    p, lse = _softmax(torch.matmul(q, k.permute(0, 2, 3, 1)), seen[:, None, None])
    out = torch.matmul(p, v.transpose(1, 2)).reshape(B, -1, D).to(s["q"].dtype)
    if not c["weight"]:
        return out, lse.view(B, -1)
    more = p.sum(2).transpose(1, 2)  # [B, t, Hk]
    b, at = seen.nonzero(as_tuple=True)
    w = s["weight"].transpose(1, 2)
    pg, pl = pages[b, at], places[b, at]
    w[pg, pl] = w[pg, pl] + more[b, at]
    return out, lse.view(B, -1), s["weight"]


def run(s):
    c = s["case"]
    if not own:
        return {"prefill": _plain_prefill, "attend": _plain_attend, "read": _plain_read}[c["op"]](s)
    cache = s["cache"]
    if c["op"] == "prefill":
        return cache.prefill(s["q"], s["starts"], s["table"], s["lengths"], window=c["window"], first=c["first"],
                             return_lse=True)
    if c["op"] == "attend":
        out, lse = cache.attend(s["q"], s["table"], s["lengths"], window=c["window"], first=c["first"],
                                add_weight=c["weight"], return_lse=True)
        return (out, lse, cache.weight) if c["weight"] else (out, lse)
    return cache.read(s["slots"], dtype=DTYPES[c["to"]])


# ------------------------------------------------------------------------------------------------- what it takes
def _visible(case, length, new):
    """Keys that at least one of the newest `new` queries sees, and (query, key) pairs."""
    window, first = case.get("window", 0), case.get("first", 0)
    if not window:
        return length, new * length - new * (new - 1) // 2
    pairs = sum(p + 1 if p + 1 <= window else window + min(first, p + 1 - window) for p in range(length - new, length))
    low = max(0, length - new - window + 1)
    return length - low + min(first, low), pairs


def work(case):
    Hk, D, size = case["kv_heads"], case["head_dim"], SIZES[case["cache"]]
    news, lengths = _lengths(case)
    if case["op"] == "read":
        return {"bytes": sum(lengths) * (Hk * D * 2 * (size + 2) + 8), "flops": 2 * sum(lengths) * Hk * D}
    H = case["heads"]
    news = news if case["op"] == "prefill" else [1] * len(lengths)
    keys, pairs = (sum(x) for x in zip(*(_visible(case, n, m) for n, m in zip(lengths, news))))
    more = keys * Hk * 8 if case.get("weight") else 0
    return {"bytes": keys * Hk * D * 2 * size + sum(news) * H * (4 * D + 4) + more + 4 * (keys // case["page"] + 2 * len(news)),
            "flops": 4 * pairs * H * D}


# ------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    page, Hk, D = case["page"], case["kv_heads"], case["head_dim"]
    wide = torch.float64

    def values(name, pages, places):
        x = _rows(s[name + "_cache"], pages, places, wide)
        return x if s[name + "_scale"] is None else x * s[name + "_scale"].to(wide).view(-1, 1)

    if case["op"] == "read":
        at = torch.div(s["slots"], page, rounding_mode="floor")
        return values("k", at, s["slots"] - at * page), values("v", at, s["slots"] - at * page)
    n = s["q"].shape[0]
    out = torch.zeros(n, case["heads"], D, dtype=wide, device="cuda")
    lse = torch.zeros(n, case["heads"], dtype=wide, device="cuda")
    weight = s["weight"].to(wide) if s["weight"] is not None else None
    starts = s["starts"].tolist() if case["op"] == "prefill" else list(range(n + 1))
    group = case["heads"] // Hk
    for r, length in enumerate(s["lengths"].tolist()):
        t = torch.arange(length, device="cuda")
        pages = s["table"][r].long()[t // page]
        k, v = values("k", pages, t % page), values("v", pages, t % page)
        for i0 in range(starts[r], starts[r + 1], 1024):
            i1 = min(starts[r + 1], i0 + 1024)
            p = torch.arange(i0, i1, device="cuda")[:, None] + (length - starts[r + 1])
            hidden = t[None, :] > p
            if case["window"]:
                hidden |= (t[None, :] <= p - case["window"]) & (t[None, :] >= case["first"])
            for h in range(Hk):
                q = s["q"][i0:i1, h * group:(h + 1) * group].to(wide)
                a = torch.einsum("igd,td->igt", q, k[:, h]) / math.sqrt(D)
                a[hidden[:, None, :].expand_as(a)] = -math.inf
                z = torch.logsumexp(a, -1)
                a = torch.exp(a - z[..., None])
                out[i0:i1, h * group:(h + 1) * group] = torch.einsum("igt,td->igd", a, v[:, h])
                lse[i0:i1, h * group:(h + 1) * group] = z
                if weight is not None:
                    weight[pages, h, t % page] += a.sum((0, 1))
    return (out, lse) if weight is None else (out, lse, weight)
