"""Plain 64-bit forms of the paged cache's operators, token by token from their definitions, for the tests."""
from __future__ import annotations

import math

import torch

DT = {"f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float8_e4m3fn: 2.0 ** -4}   # rounding to nearest
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0, torch.float8_e4m3fn: 2.0 ** -10}        # half a subnormal step


def wide(x):
    """float64 values of a tensor of any of the element types."""
    return x.float().double()


def make_pool(gen, n_pages, page, n_kv, head_dim, cache, heads_first=False, device="cuda"):
    shape = (n_pages, n_kv, page, head_dim) if heads_first else (n_pages, page, n_kv, head_dim)
    x = torch.randn(shape, generator=gen, device=device).to(DT[cache])
    return x.transpose(1, 2) if heads_first else x


def make_table(gen, lengths, page, n_pages, cols=None, fill=-1):
    """Distinct random pages for every request; entries that no token reaches are `fill`."""
    need = [-(-n // page) for n in lengths]
    cols = max([1] + need) if cols is None else cols
    order = torch.randperm(n_pages, generator=gen, device="cuda").tolist()
    assert sum(need) <= n_pages
    t = torch.full((len(lengths), cols), fill, dtype=torch.int32)
    at = 0
    for r, k in enumerate(need):
        t[r, :k] = torch.tensor(order[at:at + k], dtype=torch.int32)
        at += k
    return t.cuda(), order[at:]


def rows(pool, table_row, n, page, start=0):
    t = torch.arange(start, n, device=pool.device)
    x = pool.view(torch.uint8) if pool.dtype == torch.float8_e4m3fn else pool
    x = x[table_row.long()[t // page], t % page]
    return wide(x.view(torch.float8_e4m3fn) if pool.dtype == torch.float8_e4m3fn else x)


def ref_attend(cache, q, table, lengths, scale=None, window=0):
    """(out, lse, per-token weights as a list of [n_kv, n]), and for the bounds: sum p |v| like out, the largest
    scale * sum |q_d k_d| of each request and head."""
    B, H, D = q.shape
    Hk, page = cache.n_kv_heads, cache.page_size
    scale = 1 / math.sqrt(D) if scale is None else scale
    out = torch.zeros(B, H, D, dtype=torch.float64, device=q.device)
    mag, lse = torch.zeros_like(out), torch.full((B, H), -math.inf, dtype=torch.float64, device=q.device)
    reach = torch.zeros(B, H, dtype=torch.float64, device=q.device)
    weights = []
    for r, n in enumerate(lengths):
        start = max(0, n - window) if window else 0
        if n == 0:
            weights.append((0, None))
            continue
        k, v = rows(cache.k, table[r], n, page, start), rows(cache.v, table[r], n, page, start)
        if cache.k_scale is not None:
            k, v = k * cache.k_scale.double()[:, None], v * cache.v_scale.double()[:, None]
        x = wide(q[r]).view(Hk, H // Hk, D)
        s = torch.einsum("hgd,thd->hgt", x, k) * scale
        reach[r] = (torch.einsum("hgd,thd->hgt", x.abs(), k.abs()).amax(-1) * abs(scale)).reshape(H)
        top = s.amax(-1, keepdim=True)
        e = torch.exp(s - top)
        p = e / e.sum(-1, keepdim=True)
        out[r] = torch.einsum("hgt,thd->hgd", p, v).reshape(H, D)
        mag[r] = torch.einsum("hgt,thd->hgd", p, v.abs()).reshape(H, D)
        lse[r] = (top[..., 0] + torch.log(e.sum(-1))).reshape(H)
        weights.append((start, p.sum(1)))
    return out, lse, weights, mag, reach


def assert_attend(cache, q, table, lengths, got, lse, weight_before=None, **kw):
    """Bounds.  A logit is a sum of D products in 32 bits: D * 2^-23 of sum |q k| at most, and 2^-21 of its size for
    the scaling and the exponential.  Each softmax weight may be rounded once to q's type before it meets v, and the
    result is rounded once: unit * (|out| + sum p |v|); the rest of the sum is in 32 bits."""
    ref, rlse, rweights, mag, reach = ref_attend(cache, q, table, lengths, **kw)
    D = q.shape[2]
    unit = UNIT[q.dtype]
    logit = D * 2.0 ** -23 * reach + 2.0 ** -21 * (1 + reach)
    tol = unit * (ref.abs() + mag) + 2 * logit[..., None] * mag + 2.0 ** -16 * mag + TINY[q.dtype]
    err = (wide(got) - ref).abs()
    assert bool((err <= tol).all()), f"out off by {float((err / tol.clamp(min=1e-300)).max()):.3g} of its bound"
    live = torch.isfinite(rlse)
    assert bool((lse[~live] == -math.inf).all()) and bool((got[~live] == 0).all())
    err = (lse.double() - rlse)[live].abs()
    assert bool((err <= (logit + 2.0 ** -21 * (1 + rlse.abs()))[live]).all()), float(err.max())
    if weight_before is None:
        return
    want = weight_before.double().clone()
    slack = want.abs() * 2.0 ** -23
    page, group = cache.page_size, q.shape[1] // cache.n_kv_heads
    for r, n in enumerate(lengths):
        start, w = rweights[r]
        if w is None:
            continue
        t = torch.arange(start, n, device=q.device)
        pg, pl = table[r].long()[t // page], t % page
        want[pg, :, pl] += w.T
        worst = logit[r].view(cache.n_kv_heads, group).amax(1)
        slack[pg, :, pl] += w.T * (4 * worst[None, :] + 2.0 ** -20) + 2.0 ** -23 * want[pg, :, pl].abs()
    err = (cache.weight.double() - want).abs()
    assert bool((err <= slack).all()), f"weights off by {float((err - slack).max()):.3g} too much"


def ref_append(x, w, rope, positions, interleaved, eps):
    """float64 result for one of q, k: [n, heads, D], and the size of each row (for the bounds)."""
    x = wide(x)
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * wide(w)
    size = x.abs().amax(-1, keepdim=True)
    if rope is not None:
        r = rope.shape[1]
        half = r // 2
        row = rope.double()[positions.long()]
        y = x.clone()
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            c, s = row[:, None, i], row[:, None, half + i]
            y[..., a] = x[..., a] * c - x[..., b] * s
            y[..., b] = x[..., b] * c + x[..., a] * s
        x = y
    return x, size


def ref_evict(weight_rows, n, budget, recent, first):
    """The kept indices of one kv head, from the rule itself: weight_rows is a list of n floats."""
    keep = min(n, budget)
    recent = min(recent, budget)
    first = min(first, budget - recent)

    def rank(i):
        sure = i < first or i >= n - recent
        w = weight_rows[i]
        nan = w != w
        return (0 if sure else 1, nan, 0.0 if nan else -w, i)
    return sorted(sorted(range(n), key=rank)[:keep])
