"""Values and calls at which prefill can lose precision or go wrong, against plain 64-bit forms."""
import math
import threading

import pytest
import torch

from kv_common import DT, TINY, UNIT, make_table, wide
from kv_prompt_common import assert_prompt, ref_prompt
from paper_2604_11001_b200 import kvcache as kv
from test_kv_gpu import gen, make_cache, randn
from test_kv_values import PAGE, one_hot, stored, to_int

pytestmark = pytest.mark.gpu

# 16 and 64: pages that come in bulk; 12: row by row
TYPES = [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")]
# A softmax weight meets v in two parts: the first is at most two steps of its type below the weight, and the second, the rest, is rounded.
PARTS = {torch.bfloat16: 2.0 ** -14, torch.float16: 2.0 ** -20}


def starts_of(new):
    x = [0]
    for n in new:
        x.append(x[-1] + n)
    return x


def prefill_within(c, q, new, table, lengths, slack, **kw):
    """`new` rows of each request (all of them q[r]) within half a step of the output's type, a weight's parts and `slack` of sum p |v|; and,
    of f16, a weight's smallest step, 2^-38 of the row's largest weight, which it is half of off (twice: of both ends)."""
    q = q[:, None].expand(-1, new, -1, -1).reshape(-1, *q.shape[1:])
    starts = starts_of([new] * len(lengths))
    out, lse = c.prefill(q, to_int(starts), table, to_int(lengths), return_lse=True, **kw)
    c.check()
    ref, rlse, mag, _ = ref_prompt(c, q, starts, table, lengths, **kw)
    slack = slack + PARTS[q.dtype]
    tol = UNIT[q.dtype] * ref.abs() + (1 + UNIT[q.dtype]) * slack * mag + TINY[q.dtype]
    if q.dtype == torch.float16:
        top = c.v.float().abs().nan_to_num().amax((0, 1)).double() * (1 if c.v_scale is None else c.v_scale.double().abs()[:, None])
        tol = tol + 2.0 ** -38 * max(lengths) * top.repeat_interleave(q.shape[1] // c.n_kv_heads, 0)
    err = (out.double() - ref).abs()
    assert bool((err <= tol).all()), f"off by {float((err / tol.clamp(min=1e-300)).max()):.3g} of the bound, {int((err > tol).sum())} of {err.numel()}"
    assert bool(((lse.double() - rlse).abs() <= 2.0 ** -20 * (1 + rlse.abs()) + slack).all())
    return out, lse


# ------------------------------------------------------------------------------------------ precision
@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("gap", [6, 12, 18])
@pytest.mark.parametrize("requests,n,at,new", [(1, 40, 0, 3), (1, 5000, 0, 70), (1, 5000, 2500, 400), (2, 700, 300, 350), (30, 40, 7, 9)])
def test_one_token_far_above_the_rest(dtype, cache, gap, requests, n, at, new):
    """A token that draws nearly all of the attention and whose value is zero: the output is what the others add up to.  Exponentials: 2^-22
    of their argument at most, gap and reference (24 bits) together."""
    g = gen(gap + n)
    H, D = 2, 64
    x = 0.25 * torch.randn(requests, n, H, generator=g, device="cuda")
    x[:, at] = gap
    v = 0.5 + torch.rand(requests, n, H, D, generator=g, device="cuda")
    v[:, at] = 0
    c, q, table, lengths = one_hot(x, v, dtype, cache, 4)
    prefill_within(c, q, new, table, lengths, 2.0 ** -21 * (gap + 26), scale=1.0)


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("n,new", [(40, 1), (600, 30), (4000, 300)])
def test_a_weight_before_one_far_above_it(cache, n, new):
    """A token at e^40, the only one whose value is not zero, many at e^0, then one at e^88 that the last rows see: theirs is e^-48 of the first
    one's value."""
    g = gen(7)
    H, D = 2, 64
    x = 0.25 * torch.randn(20, n, H, generator=g, device="cuda")
    v = torch.zeros(20, n, H, D, device="cuda")
    x[:, 9], x[:, n - 5] = 40, 88
    v[:, 9] = 0.5 + torch.rand(20, H, D, generator=g, device="cuda")
    c, q, table, lengths = one_hot(x, v, "bf16", cache, 4)
    prefill_within(c, q, new, table, lengths, 2.0 ** -21 * 114, scale=1.0)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("heads_first", [False, True])
def test_logits_that_spread_over_many_powers_of_e(dtype, cache, D, heads_first):
    """Random rows with scale 1: weights from one down to e^-80."""
    g = gen(D)
    lengths, new = [700, 3, 129, 1500], [300, 3, 1, 17]
    c = make_cache(g, 160, PAGE, 2, D, cache, heads_first)
    table, _ = make_table(g, lengths, PAGE, 160)
    starts = starts_of(new)
    q = randn(g, starts[-1], 8, D, dtype=DT[dtype])
    out, lse = c.prefill(q, to_int(starts), table, to_int(lengths), return_lse=True, scale=1.0)
    c.check()
    assert_prompt(c, q, starts, table, lengths, out, lse, scale=1.0)


@pytest.mark.parametrize("n", [2, 33, 1000, 20000])
@pytest.mark.parametrize("rise", [0.0, 5.0])
def test_values_at_the_end_of_bf16(n, rise):
    """Values of 3e38: their mean is as large, and a sum of two of them is not finite."""
    g = gen(n)
    x = rise * torch.arange(n, device="cuda")[None, :, None] / n + torch.zeros(2, n, 2, device="cuda")
    v = 3e38 * (0.75 + 0.25 * torch.rand(2, n, 2, 64, generator=g, device="cuda"))
    c, q, table, lengths = one_hot(x, v, "bf16", "bf16")
    prefill_within(c, q, min(n, 150), table, lengths, 2.0 ** -16, scale=1.0)


@pytest.mark.parametrize("small", [1e-20, 1e-28])
def test_small_bf16_values_keep_their_precision(small):
    g = gen(4)
    x = torch.randn(3, 500, 2, generator=g, device="cuda")
    v = small * (1 + torch.rand(3, 500, 2, 64, generator=g, device="cuda"))
    c, q, table, lengths = one_hot(x, v, "bf16", "bf16")
    prefill_within(c, q, 200, table, lengths, 2.0 ** -16, scale=1.0)


@pytest.mark.parametrize("scale", [0.0, 1e-39, -1e-39, 1e-38, 3e-42])
def test_scales_near_zero_over_keys_at_the_end_of_bf16(scale):
    """Keys of +-3e38: their products with a scale of nearly nothing are small, their differences are not finite."""
    g = gen(3)
    x = 3e38 * torch.sign(torch.randn(3, 90, 2, generator=g, device="cuda"))
    c, q, table, lengths = one_hot(x, torch.randn(3, 90, 2, 64, generator=g, device="cuda"), "bf16", "bf16")
    prefill_within(c, q, 40, table, lengths, 2.0 ** -16, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("scale", [None, -0.3, 0.0])
@pytest.mark.parametrize("page", [12, 16])
def test_scales_of_either_sign(dtype, scale, page):
    g = gen(page)
    c = make_cache(g, 70, page, 5, 64, "e4m3")
    c.k_scale.copy_(torch.tensor([0.7, -0.4, 1.5, -2.0, 0.0]))
    c.v_scale.copy_(torch.tensor([-1.0, 0.5, 0.25, -0.75, 3.0]))
    lengths, new = [90, 300, 5], [60, 200, 5]
    table, _ = make_table(g, lengths, page, 70)
    starts = starts_of(new)
    q = randn(g, starts[-1], 15, 64, dtype=DT[dtype])
    out, lse = c.prefill(q, to_int(starts), table, to_int(lengths), return_lse=True, scale=scale)
    c.check()
    assert_prompt(c, q, starts, table, lengths, out, lse, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", [60, 1900])
@pytest.mark.parametrize("head_dim", [64, 256])
def test_a_scale_that_is_no_number_shows(dtype, n, head_dim):
    """In one piece, in several, by one tile of rows and by two."""
    one = torch.ones(2, device="cuda")
    pages = -(-n // PAGE)
    ones = torch.ones(pages, PAGE, 2, head_dim, device="cuda")
    c = kv.PagedKV(stored(ones, "e4m3"), stored(ones, "e4m3"), None, torch.tensor([float("nan"), 1.0], device="cuda"), one)
    q = torch.ones(20, 4, head_dim, device="cuda").to(DT[dtype])
    out, lse = c.prefill(q, to_int([0, 20]), torch.arange(pages, dtype=torch.int32, device="cuda")[None], to_int([n]), return_lse=True)
    assert bool(torch.isnan(out[:, :2]).all()) and bool(torch.isnan(lse[:, :2]).all())
    assert bool((out[:, 2:] == 1).all()) and bool(torch.isfinite(lse[:, 2:]).all())


# ------------------------------------------------------------------------------------------ what is seen, and what is not
def poison(c, page, place, k=None, v=None, element=slice(None)):
    for pool, x in ((c.k, k), (c.v, v)):
        if x is None:
            continue
        if pool.dtype == torch.float8_e4m3fn:
            pool.view(torch.uint8)[page, place, :, element] = 0x7f    # (it has no infinity)
        else:
            pool[page, place, :, element] = x


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("head_dim,page", [(64, 16), (128, 12), (128, 64), (256, 16), (80, 7)])
@pytest.mark.parametrize("what", ["k", "v", "both"])
def test_what_a_row_does_not_see_may_hold_anything(dtype, cache, head_dim, page, what):
    """Tokens of NaN and infinities among the new ones: rows before them, and those whose window is behind them, are as without."""
    g = gen(head_dim)
    length, new, window, first = 700, 500, 60, 9
    c = make_cache(g, 700 // page + 4, page, 2, head_dim, cache)
    table, _ = make_table(g, [length], page, c.n_pages)
    q = randn(g, new, 4, head_dim, dtype=DT[dtype])
    bad = length - new + 250
    for i, x in ((0, float("nan")), (1, float("inf")), (2, -float("inf"))):
        t = bad + i
        poison(c, int(table[0, t // page]), t % page, x if what != "v" else None, x if what != "k" else None)
    for kw, behind in ((dict(), None), (dict(window=window, first=first), 250 + 3 + window - 1)):
        out, lse = c.prefill(q, to_int([0, new]), table, to_int([length]), return_lse=True, **kw)
        c.check()
        assert_prompt(c, q[:250], [0, 250], table, [bad], out[:250], lse[:250], **kw)
        if cache == "e4m3" or what != "k":      # (a key of -infinity in places, with a q of both signs: NaN)
            assert bool(torch.isnan(out[252:250 + window]).all())
        if behind:
            assert_prompt(c, q[behind:], [0, new - behind], table, [length], out[behind:], lse[behind:], **kw)
            assert bool(torch.isfinite(out[behind:]).all())
        else:
            assert bool(torch.isnan(out[252:]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("page", [12, 16])
@pytest.mark.parametrize("new", [40, 300])
def test_infinite_values_stay_in_their_element(dtype, page, new):
    g = gen(new)
    c = make_cache(g, 60, page, 2, 64, dtype)
    length = 400
    table, _ = make_table(g, [length], page, 60)
    q = randn(g, new, 8, 64, dtype=DT[dtype])
    clean = c.prefill(q, to_int([0, new]), table, to_int([length]))
    t = length - 20                        # seen by the last 20 rows, in a tile that is not seen whole
    c.v[int(table[0, t // page]), t % page, 1, 5] = -math.inf
    c.v[int(table[0, 3]), 2, 0, 7] = math.inf   # and by all rows
    c.v[int(table[0, 4]), 2, 0, 8], c.v[int(table[0, 5]), 2, 0, 8] = math.inf, -math.inf
    out = c.prefill(q, to_int([0, new]), table, to_int([length]))
    seen = torch.arange(new, device="cuda") >= new - 20
    t3 = torch.arange(length - new, length, device="cuda")
    assert bool((out[seen][:, 4:, 5] == -math.inf).all())
    assert bool((out[t3 >= 3 * page + 2][:, :4, 7] == math.inf).all()) and bool(torch.isnan(out[t3 >= 5 * page + 2][:, :4, 8]).all())
    for got, was in ((out[~seen][:, 4:], clean[~seen][:, 4:]), (out[..., :5], clean[..., :5]), (out[..., 9:], clean[..., 9:])):
        assert torch.equal(got, was)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_infinite_keys_and_queries(dtype):
    """A logit of -infinity counts as no token, one of infinity gives NaN; those of other rows and heads stay."""
    g = gen(8)
    c = make_cache(g, 12, 16, 1, 64, dtype)
    table = torch.arange(12, device="cuda", dtype=torch.int32)[None]
    q = randn(g, 100, 2, 64, dtype=DT[dtype]).abs() + 0.1
    c.k[:5] = -math.inf                                               # the first 80 tokens: whole tiles and a part of one
    out, lse = c.prefill(q, to_int([0, 100]), table, to_int([190]), return_lse=True)
    want, wlse = c.prefill(q, to_int([0, 100]), table[:, 5:], to_int([110]), return_lse=True)
    assert_prompt(c, q, [0, 100], table[:, 5:], [110], out, lse)
    assert_prompt(c, q, [0, 100], table[:, 5:], [110], want, wlse)
    out, lse = c.prefill(q, to_int([0, 30]), table, to_int([80]), return_lse=True)
    assert bool((out[:30] == 0).all()) and bool((lse == -math.inf).all())
    q[40, 1, 3], q[41, 0] = math.inf, math.nan
    out2 = c.prefill(q, to_int([0, 100]), table[:, 5:], to_int([110]))
    assert bool(torch.isnan(out2[40, 1]).all()) and bool(torch.isnan(out2[41, 0]).all())
    rest = torch.ones(100, 2, dtype=torch.bool, device="cuda")
    rest[40, 1] = rest[41, 0] = False
    assert torch.equal(out2[rest], want[rest])
    c.check()


@pytest.mark.parametrize("cache", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("requests,n,new", [(1, 3, 2), (1, 9000, 40), (20, 100, 100), (150, 200, 1), (5, 900, 700)])
def test_rows_whose_logits_are_all_minus_infinity(cache, requests, n, new):
    H, D = 2, 64
    pages = -(-n // PAGE)
    k = torch.zeros(pages, PAGE, H, D, device="cuda")
    k[..., 0] = 1
    v = torch.randn(pages, PAGE, H, D, generator=gen(n), device="cuda")
    v[..., 3], v[..., 5] = float("nan") if cache == "e4m3" else math.inf, float("nan")
    scales = [torch.ones(H, device="cuda")] * 2 if cache == "e4m3" else [None, None]
    c = kv.PagedKV(stored(k, cache), stored(v, cache), None, *scales)
    q = torch.zeros(requests * new, 4, D, dtype=torch.float16 if cache == "f16" else torch.bfloat16, device="cuda")
    q[..., 0] = float("-inf")
    table = torch.arange(pages, dtype=torch.int32, device="cuda").expand(requests, pages).contiguous()   # (pages are only read)
    out, lse = c.prefill(q, to_int(starts_of([new] * requests)), table, to_int([n] * requests), return_lse=True)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    c.check()


# ------------------------------------------------------------------------------------------ bad pages, lengths, starts
@pytest.mark.parametrize("cache,head_dim", [("bf16", 64), ("f16", 256), ("e4m3", 128)])
@pytest.mark.parametrize("page", [7, 16, 64])
def test_bad_pages_are_left_out_and_flagged(cache, head_dim, page):
    g = gen(page)
    lengths, new = [500, 300, 40], [200, 300, 3]
    c = make_cache(g, 160, page, 2, head_dim, cache)
    table, _ = make_table(g, lengths, page, 160)
    starts = starts_of(new)
    q = randn(g, starts[-1], 4, head_dim, dtype=torch.float16 if cache == "f16" else torch.bfloat16)
    clean = c.prefill(q, to_int(starts), table, to_int(lengths))
    c.check()
    for wild in (-1, 160, 2 ** 31 - 1, -2 ** 31):
        t = table.clone()
        t[0, 1] = t[0, (500 - 1) // page] = wild
        out, lse = c.prefill(q, to_int(starts), t, to_int(lengths), return_lse=True)
        assert_prompt(c, q, starts, t, lengths, out, lse)
        assert torch.equal(out[starts[1]:], clean[starts[1]:])
        with pytest.raises(ValueError, match="page"):
            c.check()
    t = torch.full_like(table, -5)
    out, lse = c.prefill(q, to_int(starts), t, to_int(lengths), return_lse=True)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    with pytest.raises(ValueError, match="page"):
        c.check()


@pytest.mark.parametrize("requests", [4, 50])
def test_bad_lengths_and_starts_are_flagged(requests):
    g = gen(1)
    c = make_cache(g, 60, 16, 2, 64, "bf16")
    table = torch.arange(60, device="cuda", dtype=torch.int32).view(1, 60).expand(requests, 60)[:, :20].contiguous()
    lengths, new = [300, 40, 77, 5] + [9] * (requests - 4), [70, 40, 2, 0] + [1] * (requests - 4)
    starts = starts_of(new)
    n = starts[-1]
    q = randn(g, n, 4, 64, dtype=torch.bfloat16)
    run = lambda s, ln, **kw: c.prefill(q, to_int(s), table, to_int(ln), return_lse=True, **kw)  # noqa: E731

    def flagged():
        with pytest.raises(ValueError, match="length"):
            c.check()
    want, wlse = run(starts, lengths)
    c.check()
    # a length above max_length counts as max_length
    out, lse = run(starts, lengths, max_length=200)
    flagged()
    assert_prompt(c, q, starts, table, [min(x, 200) for x in lengths], out, lse)
    out, lse = run(starts, [2 ** 31 - 1] + lengths[1:])
    flagged()
    assert_prompt(c, q, starts, table, [320] + lengths[1:], out, lse)
    # fewer tokens than rows: the newest rows are the tokens, the others see nothing
    for few in (33, 0, -1, -2 ** 31):
        out, lse = run(starts, [lengths[0], few] + lengths[2:])
        flagged()
        m, none = max(few, 0), slice(starts[1], starts[2] - max(few, 0))
        assert bool((out[none] == 0).all()) and bool((lse[none] == -math.inf).all())
        assert_prompt(c, q[starts[2] - m:starts[2]], [0, m], table[1:2], [m], out[starts[2] - m:starts[2]], lse[starts[2] - m:starts[2]])
        assert torch.equal(out[:starts[1]], want[:starts[1]]) and torch.equal(out[starts[2]:], want[starts[2]:])
    # starts outside the rows count as the ends
    out, lse = run([-7] + starts[1:], lengths)
    flagged()
    assert torch.equal(out, want) and torch.equal(lse, wlse)
    out, lse = run(starts[:-1] + [2 ** 31 - 1], lengths)
    flagged()
    assert torch.equal(out, want) and torch.equal(lse, wlse)
    c.check()


# ------------------------------------------------------------------------------------------ forms of the arguments
@pytest.mark.parametrize("page", [12, 16])
@pytest.mark.parametrize("head_dim", [64, 80])
def test_strides_of_queries_and_pools(page, head_dim):
    g = gen(page)
    lengths, new = [300, 77, 140], [150, 77, 1]
    starts = starts_of(new)
    n, H = starts[-1], 6
    c = make_cache(g, 60, page, 2, head_dim, "bf16")
    table, _ = make_table(g, lengths, page, 60)
    args = to_int(starts), table, to_int(lengths)
    packed = randn(g, n, (H + 4) * head_dim, dtype=torch.bfloat16)[:, :H * head_dim].view(n, H, head_dim)
    outermost = randn(g, H, n, head_dim, dtype=torch.bfloat16).transpose(0, 1)
    behind = randn(g, n + 1, H, head_dim + 8, dtype=torch.bfloat16)[1:, :, 8:]
    for q in (packed, outermost, behind, packed[:1].expand(n, -1, -1), packed[:, :1].expand(-1, H, -1), packed[:1, :1].expand(n, H, -1), packed.flip(0)):
        out, lse = c.prefill(q, *args, return_lse=True)
        assert out.is_contiguous()
        assert_prompt(c, q, starts, table, lengths, out, lse)
    # a table of which columns are taken, and a pool whose pages are parts of larger ones
    wide_table = torch.full((3, 50), -1, dtype=torch.int32, device="cuda")
    wide_table[:, :table.shape[1]] = table
    assert torch.equal(c.prefill(packed, args[0], wide_table[:, :table.shape[1]], args[2]), c.prefill(packed, *args))
    big = [randn(g, 60, 2, page, 4, head_dim, dtype=torch.bfloat16) for _ in range(2)]
    for part in (big[0][:, 1, :, 1:3], big[1][:, 0, :, ::2]):
        d = kv.PagedKV(part, part)
        out, lse = d.prefill(packed, *args, return_lse=True)
        assert_prompt(d, packed, starts, table, lengths, out, lse)
        d.check()
    one = randn(g, 1, page, 1, head_dim, dtype=torch.bfloat16)
    for part in (one.expand(60, -1, 2, -1), one.expand(60, page, 2, head_dim)[:, :1].expand(-1, page, -1, -1)):   # the same row in many places
        d = kv.PagedKV(part, part)
        out, lse = d.prefill(packed, *args, return_lse=True)
        assert_prompt(d, packed, starts, table, lengths, out, lse)
        d.check()
    c.check()


def test_nothing_to_do():
    c = make_cache(gen(1), 4, 16, 2, 64, "f16")
    none = torch.zeros(0, 4, 64, dtype=torch.float16, device="cuda")
    out, lse = c.prefill(none, to_int([0, 0]), to_int([[0, 1]]), to_int([20]), return_lse=True)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    q = torch.ones(5, 4, 64, dtype=torch.float16, device="cuda")
    for starts, table, lengths in (([0], torch.zeros(0, 3, dtype=torch.int32, device="cuda"), to_int([])), ([2, 2, 2], to_int([[0], [1]]), to_int([0, 7]))):
        out, lse = c.prefill(q, to_int(starts), table, lengths, return_lse=True)
        assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    c.check()
    out = c.prefill(q, to_int([0, 5]), torch.zeros(1, 0, dtype=torch.int32, device="cuda"), to_int([0]))   # (five rows of a request without tokens)
    assert bool((out == 0).all())
    with pytest.raises(ValueError, match="length"):
        c.check()


@pytest.mark.parametrize("page", [16, 20])
def test_offsets_beyond_32_bits(page):
    """A pool of more than 2^32 elements, whose ends a request holds; queries and outputs of more than 2^31."""
    n_kv, D = 8, 128
    n_pages = (2 ** 32 + 2 ** 28) // (page * n_kv * D)
    k = torch.empty(n_pages, page, n_kv, D, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    g = gen(9)
    last = [0, n_pages - 1, 1, n_pages - 2, n_pages // 2 + 1]
    for p in last:
        k[p] = randn(g, page, n_kv, D).to(k.dtype)
        v[p] = randn(g, page, n_kv, D).to(k.dtype)
    c = kv.PagedKV(k, v)
    table = torch.tensor([last, last[::-1]], dtype=torch.int32, device="cuda")
    lengths, new = [77, 80], [40, 80]
    rows = 2 ** 31 // (8 * D) + 300
    q = torch.empty(rows, 8, D, dtype=torch.bfloat16, device="cuda")
    starts = [rows - 120, rows - 80, rows]
    q[starts[0]:] = randn(g, 120, 8, D).to(q.dtype)
    out, lse = c.prefill(q, to_int(starts), table, to_int(lengths), return_lse=True)
    assert_prompt(c, q[starts[0]:], [0, 40, 120], table, lengths, out[starts[0]:], lse[starts[0]:])
    assert not bool(out[:starts[0]].any()) and bool((lse[:starts[0]] == -math.inf).all())
    c.check()


def test_the_binding_refuses():
    c = make_cache(gen(1), 4, 16, 2, 64, "f16")
    q, starts, table, ln = torch.zeros(3, 4, 64, dtype=torch.float16, device="cuda"), to_int([0, 3]), to_int([[0, 1]]), to_int([20])
    ok = dict(q=q, starts=starts, table=table, lengths=ln)
    c.prefill(**ok)
    for bad in (dict(q=q.float()), dict(q=q.cpu()), dict(q=q[0]), dict(q=q[..., :32]), dict(q=torch.zeros(3, 4, 128, dtype=torch.float16, device="cuda")[..., ::2]),
                dict(q=q.bfloat16()), dict(starts=starts.long()), dict(starts=starts[:1]), dict(starts=to_int([0, 0, 3, 3])[::2]), dict(starts=starts.cpu()),
                dict(lengths=ln.long()), dict(lengths=ln.cpu()), dict(lengths=to_int([20, 20])), dict(table=table.long()), dict(table=table[0]),
                dict(table=table.cpu()), dict(table=to_int([[0, 1, 2, 3]])[:, ::2]), dict(max_length=33), dict(max_length=-1), dict(window=-1), dict(first=-1),
                dict(scale=float("nan")), dict(window=2 ** 31), dict(first=2 ** 31), dict(max_length=2 ** 40), dict(q=torch.zeros(3, 5, 64, dtype=torch.float16, device="cuda")),
                dict(q=torch.zeros(3 * 4 * 64 + 4, dtype=torch.float16, device="cuda")[4:].view(3, 4, 64))):
        with pytest.raises((ValueError, RuntimeError)):
            c.prefill(**{**ok, **bad})
    want = q.clone().requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        c.prefill(want, starts, table, ln)
    with torch.no_grad():
        assert not c.prefill(want, starts, table, ln).requires_grad
    c.check()


# ------------------------------------------------------------------------------------------ streams, graphs, threads, workspaces
def setting(seed, lengths, new, cache="bf16", heads=8):
    g = gen(seed)
    c = make_cache(g, 700, 16, 2, 128, cache)
    table, _ = make_table(g, lengths, 16, 700)
    return c, randn(g, sum(new), heads, 128, dtype=torch.bfloat16), to_int(starts_of(new)), table, to_int(lengths)


def test_calls_of_different_shapes_share_a_workspace_with_attend():
    """One cache, one stream: calls whose grids, parts and joins differ, each after another kind; what a workspace has to begin with is left so."""
    g = gen(17)
    c = make_cache(g, 2000, 16, 4, 64, "bf16")
    kinds = [([9000], [40], 16), ([40] * 200, [3] * 200, 4), ([700] * 20, [700] * 20, 32), ([1], [1], 4), ([16000], [1], 4), ([300, 5, 2000], [100, 5, 9], 64),
             ([4000] * 4, [150] * 4, 8)]
    for turn in range(2):
        for lengths, new, heads in kinds[turn:] + kinds[:turn]:
            table, _ = make_table(g, lengths, 16, 2000)
            starts = starts_of(new)
            q = randn(g, starts[-1], heads, 64, dtype=torch.bfloat16)
            out, lse = c.prefill(q, to_int(starts), table, to_int(lengths), return_lse=True)
            one = c.attend(q[:len(lengths)], table, to_int(lengths))
            again = c.prefill(q, to_int(starts), table, to_int(lengths))
            assert torch.equal(one, c.attend(q[:len(lengths)], table, to_int(lengths)))
            assert_prompt(c, q, starts, table, lengths, out, lse)
            assert torch.equal(out, again)
    assert not bool(next(iter(c._workspaces.values()))[:64 * 1024].any())
    c.check()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_on_streams_and_in_graphs(cache):
    c, q, starts, table, ln = setting(13, [3000, 1, 700, 4000], [40, 1, 700, 3], cache)
    want = c.prefill(q, starts, table, ln, return_lse=True)
    one = c.attend(q[:4], table, ln)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for i in range(12):
        with torch.cuda.stream(streams[i % 3]):
            got.append((c.prefill(q, starts, table, ln, return_lse=True), c.attend(q[:4], table, ln)))
    torch.cuda.synchronize()
    assert all(torch.equal(a[0], want[0]) and torch.equal(a[1], want[1]) and torch.equal(b, one) for a, b in got)
    graphs, outs = [], []
    for _ in range(2):    # two graphs, of two calls each, replayed on two streams at once
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            a = c.prefill(q, starts, table, ln)
            b = c.attend(q[:4], table, ln)
            d = c.prefill(q, starts, table, ln, window=100, first=4)
        graphs.append(graph), outs.append((a, b, d))
    windowed = c.prefill(q, starts, table, ln, window=100, first=4)
    torch.cuda.synchronize()
    for _ in range(5):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for a, b, d in outs:
        assert torch.equal(a, want[0]) and torch.equal(b, one) and torch.equal(d, windowed)
    # a replay reads what stands there then
    ln.copy_(to_int([2000, 1, 700, 3900])), q.copy_(q.flip(0))
    graphs[0].replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0][0], c.prefill(q, starts, table, ln))
    c.check()


def test_threads_with_caches_of_their_own_share_a_stream():
    sets = [setting(i, [900 + 100 * i, 40, 3000], [300, 40, 5 + i]) for i in range(3)]
    want = [c.prefill(*args) for c, *args in sets]
    torch.cuda.synchronize()
    wrong = []

    def run(i):
        c, *args = sets[i]
        for _ in range(20):
            if not torch.equal(c.prefill(*args), want[i]):
                wrong.append(i)
    threads = [threading.Thread(target=run, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
    for c, *_ in sets:
        c.check()


def test_a_wait_that_was_given_up_shows_and_leaves_no_workspace():
    """(The bit is set from here: no wait runs out.)"""
    c, *args = setting(3, [700, 40], [30, 40])
    want = c.prefill(*args)
    assert c._workspaces
    c.status.fill_(kv.STUCK | kv.BAD_PAGE)
    with pytest.raises(RuntimeError, match="given up"):
        c.check()
    assert not c._workspaces
    assert torch.equal(c.prefill(*args), want)
    c.check()


def test_requests_that_claim_the_same_rows_are_flagged():
    """Rows of two requests hold the output of one of them, the other rows their own."""
    c, q, starts, table, ln = setting(4, [100, 200, 300], [20, 20, 20])
    out = c.prefill(q, to_int([0, 40, 20, 60]), table, ln)     # requests of 40, none and 40 rows
    with pytest.raises(ValueError, match="length"):
        c.check()
    first = c.prefill(q[:40], to_int([0, 40]), table[:1], ln[:1])
    last = c.prefill(q[20:], to_int([0, 40]), table[2:], ln[2:])
    unit, tiny = 2.0 ** -6, 2.0 ** -6    # (other tiles, other order of sums: a step of the type or two of values below 4)
    near = lambda a, b: bool(((a.double() - b.double()).abs() <= unit * b.double().abs() + tiny).all())  # noqa: E731
    assert near(out[:20], first[:20]) and near(out[40:], last[20:])
    for i in range(20):
        for h in range(q.shape[1]):
            assert near(out[20 + i, h], first[20 + i, h]) or near(out[20 + i, h], last[i, h])


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_a_first_call_under_capture(cache):
    """Nothing is set up by a call before: what a kernel needs once is set under capture too."""
    c, q, starts, table, ln = setting(6, [900, 33], [300, 33], cache)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        out = c.prefill(q, starts, table, ln)
        k, v = c.read(torch.arange(40, device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, c.prefill(q, starts, table, ln)) and torch.equal(k, c.read(torch.arange(40, device="cuda"))[0])
    c.check()


# ------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("cache,page", [("bf16", 16), ("f16", 24), ("e4m3", 64)])
@pytest.mark.parametrize("window,first", [(0, 0), (100, 4)])
def test_prompts_in_chunks_then_tokens_then_evicted_then_moved(cache, page, window, first):
    """What a slot does: two prompts come in chunks, some tokens follow one by one, the cache is cut, read and stored elsewhere."""
    g = gen(page)
    dtype = torch.float16 if cache == "f16" else torch.bfloat16
    H, Hk, D, total = 8, 2, 64, [300, 170]
    c = make_cache(g, 2 * (400 // page + 2), page, Hk, D, cache)
    c.weight.zero_()
    cols = 400 // page + 1
    table = torch.randperm(2 * cols, generator=g, device="cuda").to(torch.int32).view(2, cols)
    rope = torch.randn(400, D // 2, generator=g, device="cuda")
    rope = torch.cat([rope.cos(), rope.sin()], 1).contiguous()
    lengths = [0, 0]
    kw = dict(window=window, first=first)

    def slots_of(r, t):
        return table[r].long()[t // page] * page + t % page

    for new in ([100, 64], [1, 106], [199, 0]):
        starts = starts_of(new)
        x = randn(g, starts[-1], H + 2 * Hk, D, dtype=dtype)
        t = [torch.arange(lengths[r], lengths[r] + new[r], device="cuda") for r in range(2)]
        q = c.append(x[:, :H], x[:, H:H + Hk], x[:, H + Hk:], torch.cat(t).int(), torch.cat([slots_of(r, t[r]) for r in range(2)]), rope=rope)
        lengths = [lengths[r] + new[r] for r in range(2)]
        out, lse = c.prefill(q, to_int(starts), table, to_int(lengths), return_lse=True, **kw)
        assert_prompt(c, q, starts, table, lengths, out, lse, **kw)
    assert lengths == total
    for _ in range(5):
        x = randn(g, 2, H + 2 * Hk, D, dtype=dtype)
        t = to_int(lengths)
        q = c.append(x[:, :H], x[:, H:H + Hk], x[:, H + Hk:], t, torch.cat([slots_of(r, t[r:r + 1]) for r in range(2)]), rope=rope)
        lengths = [n + 1 for n in lengths]
        out, lse = c.attend(q, table, to_int(lengths), add_weight=True, return_lse=True, **kw)
        assert_prompt(c, q, [0, 1, 2], table, lengths, out, lse, **kw)
        # the same rows as prompts of one token
        out, lse = c.prefill(q, to_int([0, 1, 2]), table, to_int(lengths), return_lse=True, **kw)
        assert_prompt(c, q, [0, 1, 2], table, lengths, out, lse, **kw)
    spare = make_cache(g, c.n_pages, page, Hk, D, cache)
    before = [c.read(slots_of(r, torch.arange(lengths[r], device="cuda"))) for r in range(2)]
    free = [p for p in range(c.n_pages) if p not in table.tolist()[0] + table.tolist()[1]]
    assert len(free) >= 2
    n, kept = c.evict(table, to_int(lengths), to_int([page, page]), to_int([[free[0]], [free[1]]]), recent=4, first=2)
    assert n.tolist() == [page, page]
    for r in range(2):
        k, v = c.read(free[r] * page + torch.arange(page, device="cuda"))
        for h in range(Hk):
            assert torch.equal(k[:, h], before[r][0][kept[r, h].long(), h]) and torch.equal(v[:, h], before[r][1][kept[r, h].long(), h])
        if cache != "e4m3":
            spare.append(None, k, v, None, torch.arange(page, device="cuda"))
            assert torch.equal(spare.k[0], k) and torch.equal(spare.v[0], v)
    c.check(), spare.check()
