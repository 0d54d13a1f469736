"""Plain 64-bit form of attention of several tokens per request over a paged cache, with a window and first tokens that stay visible."""
from __future__ import annotations

import math

import torch

from kv_common import TINY, UNIT, rows, wide


def visible(n, new, window, first, device="cuda"):
    """[new, n]: which of a request's n tokens its newest `new` see."""
    t = torch.arange(n, device=device)[None, :]
    p = torch.arange(n - new, n, device=device)[:, None]
    seen = t <= p
    if window:
        seen = seen & ((t > p - window) | (t < first))
    return seen


def there(table_row, n, page, n_pages):
    """[n]: tokens whose page is in the pool."""
    t = torch.arange(n, device=table_row.device)
    at = table_row.long()[t // page]
    return (at >= 0) & (at < n_pages)


def ref_prompt(cache, q, starts, table, lengths, scale=None, window=0, first=0, add=False):
    """(out, lse), and for the bounds: sum p |v| like out and the largest scale * sum |q_d k_d| of each row and head; with `add` also
    each request's weights, [n_kv, n], and the largest of those of its rows.  Rows that belong to no request are zeros and -infinity."""
    n, H, D = q.shape
    Hk, page = cache.n_kv_heads, cache.page_size
    scale = 1 / math.sqrt(D) if scale is None else scale
    out = torch.zeros(n, H, D, dtype=torch.float64, device=q.device)
    mag, lse = torch.zeros_like(out), torch.full((n, H), -math.inf, dtype=torch.float64, device=q.device)
    reach = torch.zeros(n, H, dtype=torch.float64, device=q.device)
    weights = []
    for r, length in enumerate(lengths):
        new = starts[r + 1] - starts[r]
        if length == 0 or new == 0:
            weights.append(None)
            continue
        live = there(table[r], length, page, cache.n_pages)
        row = torch.where(torch.arange(table.shape[1], device=q.device) * page < length, table[r], 0).clamp(0, cache.n_pages - 1)
        k, v = rows(cache.k, row, length, page), rows(cache.v, row, length, page)
        if cache.k_scale is not None:
            k, v = k * cache.k_scale.double()[:, None], v * cache.v_scale.double()[:, None]
        seen = visible(length, new, window, first, q.device) & live[None, :]
        k, v = k.masked_fill(~live[:, None, None], 0), v.masked_fill(~live[:, None, None], 0)
        gone = ~seen.any(0)  # what no row sees may hold anything
        k, v = k.masked_fill(gone[:, None, None], 0), v.masked_fill(gone[:, None, None], 0)
        x = wide(q[starts[r]:starts[r + 1]]).view(new, Hk, H // Hk, D)
        s = torch.einsum("ihgd,thd->ihgt", x, k) * scale
        a = (torch.einsum("ihgd,thd->ihgt", x.abs(), k.abs()) * abs(scale)).masked_fill(~seen[:, None, None], 0)
        s = s.masked_fill(~seen[:, None, None], -math.inf)
        top = s.amax(-1, keepdim=True).clamp(min=-1e300)
        e = torch.exp(s - top)
        total = e.sum(-1, keepdim=True)
        p = e / total.clamp(min=1e-300)
        here = slice(starts[r], starts[r + 1])
        out[here] = torch.einsum("ihgt,thd->ihgd", p, v).reshape(new, H, D)
        mag[here] = torch.einsum("ihgt,thd->ihgd", p, v.abs()).reshape(new, H, D)
        lse[here] = (top + torch.log(total))[..., 0].reshape(new, H)
        reach[here] = a.amax(-1).reshape(new, H)
        weights.append(p.sum((0, 2)))
    return (out, lse, mag, reach, weights) if add else (out, lse, mag, reach)


def assert_prompt(cache, q, starts, table, lengths, got, lse, **kw):
    """Bounds.  A logit is a sum of D products in 32 bits: D * 2^-23 of sum |q k| at most, and 2^-21 of its size for the scaling
    and the exponential.  A softmax weight meets v in two 16-bit parts, 2^-15 of it off at most, and is a multiple of 2^-38 of the
    row's largest (f16); the result is rounded once; the rest of the sum is in 32 bits."""
    ref, rlse, mag, reach = ref_prompt(cache, q, starts, table, lengths, **kw)
    D = q.shape[2]
    unit = UNIT[q.dtype]
    logit = D * 2.0 ** -23 * reach + 2.0 ** -21 * (1 + reach)
    tol = unit * ref.abs() + (1 + unit) * (2 * logit[..., None] * mag + 2.0 ** -14 * mag) + TINY[q.dtype]
    err = (wide(got) - ref).abs()
    assert bool((err <= tol).all()), f"out off by {float((err / tol.clamp(min=1e-300)).max()):.3g} of its bound"
    live = torch.isfinite(rlse)
    assert bool((lse[~live] == -math.inf).all()) and bool((got[~live] == 0).all())
    err = (lse.double() - rlse)[live].abs()
    assert bool((err <= (logit + 2.0 ** -20 * (1 + rlse.abs()))[live]).all()), float(err.max()) if err.numel() else 0
