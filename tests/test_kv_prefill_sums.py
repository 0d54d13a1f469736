"""The sum of a row's weights over long contexts, where one CTA walks over all of them."""
import math

import pytest
import torch

from kv_common import DT, UNIT, wide
from paper_2604_11001_b200 import kvcache as kv
from test_kv_gpu import gen
from test_kv_prefill_values import PARTS, starts_of, to_int
from test_kv_values import stored

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("new,head_dim", [(1, 64), (200, 64), (1, 256)])
@pytest.mark.parametrize("below", [0.375, 0.6875, 1.125])
def test_the_sum_of_a_long_row(dtype, cache, new, head_dim, below):
    """One token at logit `below`, many at 0: weights that are all alike, so that roundings of their sum go the same way.  More blocks than CTAs: most are
    walked over by one CTA.  A tile's weights are added up by themselves, at most 66 additions one behind the other, and each tile's sum is one more
    addition to the row's; with a relative error of 2^-24 each, and 2^-20 * (1 + lse) for the exponential, the logarithm and the joins."""
    n, requests = 1 << 19 if new == 1 else 1 << 16, 300 if new == 1 else 150
    page, keys = 64, 128 if head_dim <= 128 else 64
    k = torch.zeros(n // page, page, 1, head_dim, device="cuda")
    k[0, 0, 0, 0] = below
    scales = [torch.ones(1, device="cuda")] * 2 if cache == "e4m3" else [None, None]
    c = kv.PagedKV(stored(k, cache), stored(torch.ones_like(k), cache), None, *scales)
    q = torch.zeros(requests * new, 1, head_dim, dtype=DT[dtype], device="cuda")
    q[..., 0] = 1
    table = torch.arange(n // page, dtype=torch.int32, device="cuda").expand(requests, -1).contiguous()   # (pages are only read)
    _, lse = c.prefill(q, to_int(starts_of([new] * requests)), table, to_int([n] * requests), scale=1.0, return_lse=True)
    c.check()
    seen = torch.arange(n - new, n, device="cuda").double() + 1
    want = torch.log(math.exp(below) + (seen - 1)).repeat(requests)
    err = float((lse[:, 0].double() - want).abs().max())
    assert err <= 2.0 ** -24 * (n / keys + 66) + 2.0 ** -20 * (1 + float(want.max())), err


@pytest.mark.parametrize("dtype,cache", [("f16", "f16"), ("f16", "e4m3"), ("bf16", "bf16")])
@pytest.mark.parametrize("new,head_dim", [(1, 64), (200, 64), (200, 128), (3, 256)])
@pytest.mark.parametrize("page", [64, 20])
def test_the_output_of_a_long_row(dtype, cache, new, head_dim, page):
    """Logits that rise in steps along 262 144 tokens (the reference moves, and what was summed up before shrinks), values of one sign.  The tensor core's
    sums lose up to 2^-23 of themselves at each of 16 additions a tile of 128 tokens (8 a tile of 64 where rows are wider); what 128 tiles add up to is
    put aside: 2^-12 of the output at most.  Besides half a step of its type, a weight's parts, and 2^-20 * 20 for logits and exponentials."""
    n, requests, H = 1 << 18, 150, 2
    n = n // page * page
    g = gen(new)
    steps = torch.tensor([0.0, 1.0, 1.5, 2.0, 2.25, 2.25, 4.5, 4.5, 5.0, 4.0, 5.0, 5.0])
    x = steps[torch.arange(n) * len(steps) // n].cuda()[:, None] + torch.tensor([0.0, 0.25], device="cuda")
    k = torch.zeros(n, H, head_dim, device="cuda")
    k[..., 0] = x
    v = 1 + torch.rand(n, H, head_dim, generator=g, device="cuda")
    pool = lambda y: stored(y.view(n // page, page, H, head_dim), cache)  # noqa: E731
    scales = [torch.ones(H, device="cuda")] * 2 if cache == "e4m3" else [None, None]
    c = kv.PagedKV(pool(k), pool(v), None, *scales)
    q = torch.zeros(requests * new, H, head_dim, dtype=DT[dtype], device="cuda")
    q[..., 0] = 1
    table = torch.arange(n // page, dtype=torch.int32, device="cuda").expand(requests, -1).contiguous()   # (pages are only read)
    args = q, to_int(starts_of([new] * requests)), table, to_int([n] * requests)
    out, lse = c.prefill(*args, scale=1.0, return_lse=True)
    c.check()
    p = torch.exp(wide(c.k).view(n, H, head_dim)[..., 0] - 8)    # (as they are stored)
    sums, total = torch.cumsum(p[..., None] * wide(c.v).view(n, H, head_dim), 0)[n - new:], torch.cumsum(p, 0)[n - new:]
    want = sums / total[..., None]
    slack = UNIT[DT[dtype]] + 2.0 ** -12 + PARTS[DT[dtype]] + 20 * 2.0 ** -20
    err = (out.double().view(requests, new, H, head_dim) / want - 1).abs().max()
    assert float(err) <= slack, (float(err), slack)
    assert float((lse.double().view(requests, new, H) - torch.log(total) - 8).abs().max()) <= 2.0 ** -24 * (n / 64 + 66) + 2.0 ** -19 * 20
    assert torch.equal(c.prefill(*args, scale=1.0), out)


@pytest.mark.parametrize("dtype,cache", [("f16", "f16"), ("bf16", "bf16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("new,head_dim", [(1, 64), (200, 64), (140, 128), (3, 256)])
@pytest.mark.parametrize("what", ["late", "far", "pages", "window"])
def test_long_rows_with_gaps(dtype, cache, new, head_dim, what):
    """Walks of more than 16 384 tokens whose first 40 000 have logits of -infinity; whose last few are far above all before; that have no page for most
    of them; that see first tokens and a window.  Bounds as above."""
    n, requests, H, page = 70000 // 16 * 16, 150, 2, 16
    g = gen(new)
    x = torch.randn(n, H, generator=g, device="cuda")
    if what == "late" and cache != "e4m3":
        x[:40000] = -math.inf
    if what == "far":
        x[n - new - 5] += 96
    k = torch.zeros(n, H, head_dim, device="cuda")
    k[..., 0] = x
    v = 1 + torch.rand(n, H, head_dim, generator=g, device="cuda")
    pool = lambda y: stored(y.view(n // page, page, H, head_dim), cache)  # noqa: E731
    scales = [torch.ones(H, device="cuda")] * 2 if cache == "e4m3" else [None, None]
    c = kv.PagedKV(pool(k), pool(v), None, *scales)
    q = torch.zeros(requests * new, H, head_dim, dtype=DT[dtype], device="cuda")
    q[..., 0] = 1
    there = torch.ones(n // page, dtype=torch.bool, device="cuda")
    if what in ("pages", "late"):
        there[:2500] = False if what == "pages" else cache != "e4m3"
        there[3100:3300] = False
    table = torch.where(there, torch.arange(n // page, device="cuda"), -1).int().expand(requests, -1).contiguous()   # (pages are only read)
    window, first = (50000, 100) if what == "window" else (0, 0)
    args = q, to_int(starts_of([new] * requests)), table, to_int([n] * requests)
    out, lse = c.prefill(*args, scale=1.0, window=window, first=first, return_lse=True)
    if bool(there.all()):
        c.check()
    else:
        with pytest.raises(ValueError, match="page"):
            c.check()
    s = wide(c.k).view(n, H, head_dim)[..., 0].masked_fill(~there.repeat_interleave(page)[:, None], -math.inf)
    top = s.max()
    w, values = torch.exp(s - top), wide(c.v).view(n, H, head_dim)
    rows = torch.arange(n - new, n, device="cuda")
    sums, total = torch.cumsum(w[..., None] * values, 0), torch.cumsum(w, 0)
    want, all_of = sums[rows], total[rows]
    if window:      # less what lies between the first tokens and the window
        want, all_of = want - sums[rows - window] + sums[first - 1], all_of - total[rows - window] + total[first - 1]
    slack = UNIT[DT[dtype]] + 2.0 ** -12 + PARTS[DT[dtype]] + 110 * 2.0 ** -20
    err = (out.double().view(requests, new, H, head_dim) / (want / all_of[..., None]) - 1).abs().max()
    assert float(err) <= slack, (float(err), slack)
    assert float((lse.double().view(requests, new, H) - torch.log(all_of) - top).abs().max()) <= 2.0 ** -24 * (n / 64 + 66) + 2.0 ** -19 * 110
    assert torch.equal(c.prefill(*args, scale=1.0, window=window, first=first), out)


def test_a_long_row_whose_logits_are_all_minus_infinity():
    n = 40000
    k = torch.full((n // 16, 16, 1, 64), -1.0, device="cuda")
    c = kv.PagedKV(stored(k, "bf16"), stored(k, "bf16"))
    q = torch.full((300, 1, 64), math.inf, dtype=torch.bfloat16, device="cuda")
    table = torch.arange(n // 16, dtype=torch.int32, device="cuda").expand(150, -1).contiguous()
    out, lse = c.prefill(q, to_int(starts_of([2] * 150)), table, to_int([n] * 150), return_lse=True)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    c.check()
