"""Values and calls at which the paged cache's operators can lose precision or go wrong, against plain 64-bit forms."""
import math

import pytest
import torch

from kv_common import DT, TINY, UNIT, assert_attend, make_table, ref_attend
from paper_2604_11001_b200 import kvcache as kv
from paper_2604_11001_b200.binding import FcsimError

pytestmark = pytest.mark.gpu

PAGE = 16


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def to_int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def stored(x, cache):
    """A pool of the cache's type that holds `x`."""
    return x.to(DT[cache])


def one_hot(logits, v, dtype, cache, heads=None, q0=1.0, **scales):
    """A cache in which token t of request r has the logit logits[r, t, h] (its key's first element; the others are zero, so that
    the product is exact) and the value v[r, t, h], queries that read them with scale 1, table and lengths."""
    B, n, H = logits.shape
    D, pages = v.shape[-1], -(-n // PAGE)
    k = torch.zeros(B * pages, PAGE, H, D, device="cuda")
    values = torch.zeros_like(k)
    t = torch.arange(n, device="cuda")
    at = torch.arange(B, device="cuda")[:, None] * pages + (t // PAGE)[None, :]
    k[at, (t % PAGE).expand(B, n), :, 0] = logits
    values[at, (t % PAGE).expand(B, n)] = v
    if cache == "e4m3":
        scales = {name: scales.get(name, torch.ones(H, device="cuda")) for name in ("k_scale", "v_scale")}
    c = kv.PagedKV(stored(k, cache), stored(values, cache), **scales)
    q = torch.zeros(B, heads or H, D, dtype=DT[dtype], device="cuda")
    q[..., 0] = q0
    table = torch.arange(B * pages, dtype=torch.int32, device="cuda").view(B, pages)
    return c, q, table, [n] * B


def attend_within(c, q, table, lengths, slack, **kw):
    """Attention within half a step of the output's type and `slack` of sum p |v|."""
    out, lse = c.attend(q, table, to_int(lengths), return_lse=True, **kw)
    c.check()
    ref, rlse, _, mag, _ = ref_attend(c, q, table, lengths, **kw)
    err = (out.double() - ref).abs()
    half_step = torch.ldexp(torch.full_like(ref, UNIT[q.dtype]), torch.frexp(ref).exponent - 1)
    tol = torch.where(ref == 0, 0, half_step) + slack * mag + TINY[q.dtype]
    assert bool((err <= tol).all()), f"off by {float((err / tol.clamp(min=1e-300)).max()):.3g} of the bound, {int((err > tol).sum())} of {err.numel()}"
    assert bool(((lse.double() - rlse).abs() <= 2.0 ** -20 * (1 + rlse.abs()) + slack).all())
    return out, lse


# ------------------------------------------------------------------------------------------ precision of attend
@pytest.mark.parametrize("dtype,cache", [("f16", "f16"), ("f16", "e4m3")])
@pytest.mark.parametrize("gap", [6, 12, 18, 30])
@pytest.mark.parametrize("requests,n,at", [(1, 40, 0), (1, 5000, 0), (1, 5000, 2500), (2, 700, 699), (300, 40, 7)])
def test_one_token_far_above_the_rest(dtype, cache, gap, requests, n, at):
    """A token that draws nearly all of the attention and whose value is zero: the output is what the others add up to, e^-gap
    of its weight each.  A weight meets v in two parts of f16 whose smallest step is 2^-24; the reference of the exponentials
    follows a tile's largest weight down to 2^-8, so the step is 2^-16 of it and a rounding 2^-17.  The logits of the others
    spread by 0.25, eight of these within a tile: 2^-14.1 of the smallest.  Exponentials: 2^-22 of their argument at most, gap
    and reference (23 bits) together."""
    g = gen(gap + n)
    H, D = 2, 64
    x = 0.25 * torch.randn(requests, n, H, generator=g, device="cuda")
    x[:, at] = gap
    v = 200 * (0.5 + torch.rand(requests, n, H, D, generator=g, device="cuda"))
    v[:, at] = 0
    c, q, table, lengths = one_hot(x, v, dtype, cache, 4)
    attend_within(c, q, table, lengths, 2.0 ** -14 + 2.0 ** -21 * (gap + 16), scale=1.0)


@pytest.mark.parametrize("gap", [6, 12, 18, 30])
@pytest.mark.parametrize("requests,n,at", [(1, 40, 0), (1, 5000, 0), (1, 5000, 2500), (2, 700, 699), (300, 40, 7)])
def test_one_token_far_above_the_rest_in_bf16(gap, requests, n, at):
    """The same where the output has bf16's range: the others' weights are exact to 2^-18 down to 2^-100 of it."""
    g = gen(gap + n)
    H, D = 2, 64
    x = 0.25 * torch.randn(requests, n, H, generator=g, device="cuda")
    x[:, at] = gap
    v = 0.5 + torch.rand(requests, n, H, D, generator=g, device="cuda")
    v[:, at] = 0
    c, q, table, lengths = one_hot(x, v, "bf16", "e4m3", 4)
    attend_within(c, q, table, lengths, 2.0 ** -17 + 2.0 ** -21 * (gap + 16), scale=1.0)


@pytest.mark.parametrize("dtype,cache", [("f16", "f16"), ("f16", "e4m3"), ("bf16", "e4m3"), ("bf16", "bf16")])
@pytest.mark.parametrize("D", [96, 128, 256])
@pytest.mark.parametrize("longest", [20, 1500])
def test_logits_that_spread_over_many_powers_of_e(dtype, cache, D, longest):
    """Random rows with scale 1: weights from one down to e^-80, and elements of v that are zero beside the largest."""
    g = gen(D + longest)
    H, requests = 4, 30
    lengths = torch.randint(0, longest + 1, (requests,), generator=g, device="cuda").tolist()
    pages = sum(-(-n // PAGE) for n in lengths) + 2
    shape = (pages, PAGE, H, D)
    scales = [0.5 + torch.rand(H, generator=g, device="cuda") if cache == "e4m3" else None for _ in range(2)]
    c = kv.PagedKV(stored(torch.randn(shape, generator=g, device="cuda"), cache),
                   stored(torch.randn(shape, generator=g, device="cuda").mul(torch.rand(shape, generator=g, device="cuda") > 0.3), cache),
                   torch.rand(pages, H, PAGE, generator=g, device="cuda"), *scales)
    table, _ = make_table(g, lengths, PAGE, pages)
    q = torch.randn(requests, 2 * H, D, generator=g, device="cuda").to(DT[dtype])
    before = c.weight.clone()
    out, lse = c.attend(q, table, to_int(lengths), add_weight=True, return_lse=True, scale=1.0)
    c.check()
    assert_attend(c, q, table, lengths, out, lse, before, scale=1.0)


@pytest.mark.parametrize("dtype,cache", [("bf16", "e4m3"), ("bf16", "bf16")])
@pytest.mark.parametrize("n", [40, 600, 4000])
def test_a_weight_before_one_far_above_it(dtype, cache, n):
    """A token at e^40, the only one whose value is not zero, many at e^0, where the reference follows them down, then one at e^88: the
    output is e^-48 of the first one's value."""
    g = gen(7)
    H, D = 2, 64
    x = 0.25 * torch.randn(20, n, H, generator=g, device="cuda")
    v = torch.zeros(20, n, H, D, device="cuda")
    x[:, 9], x[:, n - 5] = 40, 88
    v[:, 9] = 0.5 + torch.rand(20, H, D, generator=g, device="cuda")
    v[:, 9, :, ::2] = 0                                # (what is nothing yet makes the sums slight)
    c, q, table, lengths = one_hot(x, v, dtype, cache, 4)
    attend_within(c, q, table, lengths, 2.0 ** -16 + 2.0 ** -21 * 104, scale=1.0)


@pytest.mark.parametrize("gap", [6, 12, 18, 22])
@pytest.mark.parametrize("n,at", [(12, 3), (40, 0), (900, 450)])
def test_large_f16_values_below_one_token_far_above(gap, n, at):
    """f16 rows of values about 30 000: what the others add up to is well within the output's range, in that token's own tile too."""
    g = gen(gap + n)
    H, D = 2, 64
    x = 0.25 * torch.randn(8, n, H, generator=g, device="cuda")
    x[:, at] = gap
    v = 20000 * (1 + torch.rand(8, n, H, D, generator=g, device="cuda"))
    v[:, at] = 0
    c, q, table, lengths = one_hot(x, v, "f16", "f16", 4)
    attend_within(c, q, table, lengths, 2.0 ** -17 + 2.0 ** -21 * (gap + 16), scale=1.0)


def test_an_infinite_f16_value_among_small_weights():
    """The passes for small weights leave out a tile that has one, or a NaN: it stays in its element, the rest is as exact as without them."""
    H, D, n = 1, 64, 40
    x = torch.zeros(3, n, H, device="cuda")
    x[:, 5] = 12
    v = torch.ones(3, n, H, D, device="cuda")
    v[:, 5] = 0
    v[1, 9, 0, 7] = float("inf")
    v[2, 9, 0, 7] = float("nan")
    c, q, table, lengths = one_hot(x, v, "f16", "f16")
    out = c.attend(q, table, to_int(lengths), scale=1.0)
    want = 39 * math.exp(-12) / (1 + 39 * math.exp(-12))
    assert float(out[1, 0, 7]) == math.inf and bool(torch.isnan(out[2, 0, 7]))
    rest = [i for i in range(64) if i != 7]
    for r in range(3):
        # (without the passes: 2^-25 of a weight that is 2^-17.3 of 2^14, on 15 of 39)
        assert bool(((out[r, 0, rest].double() - want).abs() <= 2.0 ** -11 * want + 2.0 ** -21 * want * 29).all())
    assert bool(((out[0, 0].double() - want).abs() <= 2.0 ** -11 * want + 2.0 ** -21 * want * 29).all())


@pytest.mark.parametrize("dtype,cache", [("f16", "f16"), ("f16", "e4m3"), ("bf16", "e4m3")])
@pytest.mark.parametrize("requests", [3, 400])
def test_weights_meet_values_unrounded(dtype, cache, requests):
    check_weights(dtype, cache, requests)


def check_weights(dtype, cache, requests):
    """Two tokens, the first one's value zero: the output is the second one's weight times its value.  Logits are exact, so the weight
    is within 2^-20 (an exponent of up to 16 rounded twice, the exponential, for both tokens: 2 (2^-21 ln 2 + 2^-22.5)); its
    parts, the sum, the quotient and the product add 2^-21 at most."""
    g = gen(requests)
    H, D = 8, 64
    x = torch.zeros(requests, 2, H, device="cuda")
    x[:, 1] = (1.5 * torch.randn(requests, H, generator=g, device="cuda")).clamp(-4, 4)
    v = torch.randn(requests, 2, H, D, generator=g, device="cuda") + 2
    v[:, 0] = 0
    c, q, table, lengths = one_hot(x, v, dtype, cache)
    attend_within(c, q, table, lengths, 2.0 ** -19, scale=1.0)


@pytest.mark.parametrize("requests", [3, 400])
def test_weights_meet_bf16_values_unrounded(requests):
    check_weights("bf16", "bf16", requests)


@pytest.mark.parametrize("n", [2, 33, 1000, 20000])
@pytest.mark.parametrize("rise", [0.0, 5.0])
def test_values_at_the_end_of_bf16(n, rise):
    """Values of 3e38: their mean is as large, and a sum of two of them is not finite."""
    g = gen(n)
    x = rise * torch.arange(n, device="cuda")[None, :, None] / n + torch.zeros(2, n, 2, device="cuda")
    v = 3e38 * (0.75 + 0.25 * torch.rand(2, n, 2, 64, generator=g, device="cuda"))
    c, q, table, lengths = one_hot(x, v, "bf16", "bf16")
    attend_within(c, q, table, lengths, 2.0 ** -16, scale=1.0)


@pytest.mark.parametrize("small", [1e-20, 1e-28])
def test_small_bf16_values_keep_their_precision(small):
    g = gen(4)
    x = torch.randn(3, 500, 2, generator=g, device="cuda")
    v = small * (1 + torch.rand(3, 500, 2, 64, generator=g, device="cuda"))
    c, q, table, lengths = one_hot(x, v, "bf16", "bf16")
    attend_within(c, q, table, lengths, 2.0 ** -16, scale=1.0)


@pytest.mark.parametrize("large", [[2.0 ** 8], [2.0 ** 20, -2.0 ** 10]])
@pytest.mark.parametrize("small", [1.0, 2.0 ** -20, 2.0 ** -100, 2.0 ** 100])
def test_bf16_queries_of_a_wide_range_over_8_bits(large, small):
    """Elements of q far below the head's largest decide the logits where the keys are zero beside the large ones."""
    g = gen(len(large))
    B, n, H, D = 5, 70, 2, 64
    k = torch.randn(B * 5, PAGE, H, D, generator=g, device="cuda")
    k[..., :len(large)] = 0
    v = torch.randn(B * 5, PAGE, H, D, generator=g, device="cuda")
    one = torch.ones(H, device="cuda")
    c = kv.PagedKV(stored(k, "e4m3"), stored(v, "e4m3"), k_scale=one, v_scale=one)
    q = (small * torch.randn(B, 6, D, generator=g, device="cuda")).bfloat16()
    q[..., :len(large)] = (small * torch.tensor(large, device="cuda")).bfloat16()
    q[0, 1] = 0                                       # a head without any
    q[1, :, :len(large)] = 0                          # and one without large ones
    table = torch.arange(B * 5, dtype=torch.int32, device="cuda").view(B, 5)
    # sums of 64 products in 32 bits: 64 * 2^-23 of sum |q k|, which is below 100 here; twice, for the weight and for the sum
    attend_within(c, q, table, [n] * B, 2.0 ** -9, scale=1.0 / small)


def test_infinite_queries_over_8_bits():
    """An infinite element of q: logits of -infinity where the key has the other sign, whatever the finite elements are."""
    H, D = 1, 64
    k = torch.zeros(5, PAGE, H, D, device="cuda")
    k[..., 0] = -1
    k[..., 1] = -1
    k[2, :, :, 0] = 1
    v = torch.randn(5, PAGE, H, D, generator=gen(1), device="cuda")
    one = torch.ones(H, device="cuda")
    c = kv.PagedKV(stored(k, "e4m3"), stored(v, "e4m3"), k_scale=one, v_scale=one)
    q = torch.zeros(2, 2, D, dtype=torch.bfloat16, device="cuda")
    q[0, :, 0] = float("inf")
    q[0, :, 1] = -1e30
    q[1, :, 1] = 1
    out, lse = c.attend(q, torch.arange(5, dtype=torch.int32, device="cuda").expand(2, 5), to_int([32, 80]), return_lse=True, scale=1.0)
    assert bool((out[0] == 0).all()) and bool((lse[0] == -math.inf).all())      # all of the 32 tokens' logits are -infinity
    ref = c.v.float().double().reshape(80, D).mean(0)
    assert bool(((out[1].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -18).all())


# ------------------------------------------------------------------------------------------ scales
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("scale", [None, -0.3, 0.0])
@pytest.mark.parametrize("requests", [1, 60])
def test_scales_of_either_sign(dtype, scale, requests):
    """A stored x stands for x * scale, whatever the scale's sign: logits, log-sum-exp and added weights follow."""
    g = gen(requests)
    H, D, n = 5, 64, 90
    shape = (requests * 6, PAGE, H, D)
    k_scale = torch.tensor([0.7, -0.4, 1.5, -2.0, 0.0], device="cuda")
    v_scale = torch.tensor([-1.0, 0.5, 0.25, -0.75, 3.0], device="cuda")
    c = kv.PagedKV(stored(torch.randn(shape, generator=g, device="cuda"), "e4m3"), stored(torch.randn(shape, generator=g, device="cuda"), "e4m3"),
                   torch.rand(shape[0], H, PAGE, generator=g, device="cuda"), k_scale, v_scale)
    q = torch.randn(requests, 3 * H, D, generator=g, device="cuda").to(DT[dtype])
    table = torch.arange(shape[0], dtype=torch.int32, device="cuda").view(requests, 6)
    before = c.weight.clone()
    out, lse = c.attend(q, table, to_int([n] * requests), add_weight=True, return_lse=True, scale=scale)
    c.check()
    assert_attend(c, q, table, [n] * requests, out, lse, before, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("requests", [1, 400])
def test_a_scale_that_is_no_number_shows(dtype, requests):
    H, D = 2, 64
    shape = (requests, PAGE, H, D)
    c = kv.PagedKV(stored(torch.ones(shape, device="cuda"), "e4m3"), stored(torch.ones(shape, device="cuda"), "e4m3"),
                   torch.zeros(requests, H, PAGE, device="cuda"), torch.tensor([float("nan"), 1.0], device="cuda"), torch.ones(H, device="cuda"))
    q = torch.ones(requests, 4, D, device="cuda").to(DT[dtype])
    table = torch.arange(requests, dtype=torch.int32, device="cuda").view(requests, 1)
    out, lse = c.attend(q, table, to_int([9] * requests), add_weight=True, return_lse=True)
    for x in (out[:, :2], lse[:, :2], c.weight[:, 0, :9]):
        assert bool(torch.isnan(x).all())
    assert bool((out[:, 2:] == 1).all()) and bool(torch.isfinite(lse[:, 2:]).all()) and bool(torch.isfinite(c.weight[:, 1]).all())


@pytest.mark.parametrize("scale", [0.0, 1e-39, -1e-39, 1e-38, 3e-42])
def test_scales_near_zero_over_keys_at_the_end_of_bf16(scale):
    """Keys of +-3e38: their products with a scale of nearly nothing are small, their differences are not finite."""
    g = gen(3)
    x = 3e38 * torch.sign(torch.randn(3, 90, 2, generator=g, device="cuda"))
    c, q, table, lengths = one_hot(x, torch.randn(3, 90, 2, 64, generator=g, device="cuda"), "bf16", "bf16")
    # a scale of 1e-39 has 20 bits, one of 3e-42 11, and logits of 0.3 and 0.001; the smallest unit is 2^-149, 5e-7 of a logit here
    attend_within(c, q, table, lengths, 2.0 ** -16, scale=scale)


# ------------------------------------------------------------------------------------------ nothing left, by every division
@pytest.mark.parametrize("cache", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("requests,n", [(1, 3), (1, 9000), (20, 100), (60, 700), (150, 200), (700, 3), (700, 40), (300, 400)])
def test_requests_whose_logits_are_all_minus_infinity(cache, requests, n):
    """Zeros and -infinity, as without tokens, whatever the values are and however the work is divided."""
    H, D = 2, 64
    pages = -(-n // PAGE)
    k = torch.zeros(pages, PAGE, H, D, device="cuda")
    k[..., 0] = 1
    v = torch.randn(pages, PAGE, H, D, generator=gen(n), device="cuda")
    v[..., 3], v[..., 5] = float("inf"), float("nan")
    if cache == "e4m3":
        v[..., 3] = float("nan")                        # (it has no infinity)
    scales = [torch.ones(H, device="cuda")] * 2 if cache == "e4m3" else [None, None]
    c = kv.PagedKV(stored(k, cache), stored(v, cache), None, *scales)
    q = torch.zeros(requests, 4, D, dtype=torch.float16 if cache == "f16" else torch.bfloat16, device="cuda")
    q[..., 0] = float("-inf")
    table = torch.arange(pages, dtype=torch.int32, device="cuda").expand(requests, pages).contiguous()   # (pages are only read)
    out, lse = c.attend(q, table, to_int([n] * requests), return_lse=True)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    c.check()


# ------------------------------------------------------------------------------------------ evict
@pytest.mark.parametrize("n,budget", [(40, 24), (1500, 900)])
@pytest.mark.parametrize("recent,first", [(0, 0), (10, 10)])
def test_evicted_rows_of_a_bad_page_are_zero(n, budget, recent, first):
    """Tokens of a page outside the pool rank as NaN does; those that are kept become rows of zeros, not what the page held before."""
    g = gen(n)
    pages, cols, new_cols = 200, -(-n // PAGE), -(-budget // PAGE)
    c = kv.PagedKV(torch.randn(pages, PAGE, 2, 64, generator=g, device="cuda").half(), torch.randn(pages, PAGE, 2, 64, generator=g, device="cuda").half(),
                   torch.rand(pages, 2, PAGE, generator=g, device="cuda") + 1)
    table = torch.arange(cols, dtype=torch.int32, device="cuda")[None].clone()
    new = torch.arange(pages - new_cols, pages, dtype=torch.int32, device="cuda")[None].clone()
    for wild in range(0, cols, 2):                     # half of the pages, the first among them: some must be kept
        table[0, wild] = pages + wild
    if cols % 2 == 0:
        table[0, -1] = -1
    k0, v0, w0 = c.k.clone(), c.v.clone(), c.weight.clone()
    got, kept = c.evict(table, to_int([n]), to_int([budget]), new, recent=recent, first=first)
    with pytest.raises(ValueError, match="page"):
        c.check()
    assert got.tolist() == [budget]
    row = torch.arange(budget, device="cuda")
    a, b = new[0].long()[row // PAGE], row % PAGE
    bad = 0
    for h in range(2):
        old = kept[0, h, :budget].long()
        assert bool((old[1:] > old[:-1]).all()) and int(old[0]) >= 0 and int(old[-1]) < n
        page, place = table[0].long()[old // PAGE], old % PAGE
        good = (page >= 0) & (page < pages)
        bad += int((~good).sum())
        page = page.clamp(0, pages - 1)
        for pool, before in ((c.k, k0), (c.v, v0)):
            want = torch.where(good[:, None], before[page, place, h], torch.zeros(64, device="cuda").half())
            assert torch.equal(pool[a, b, h], want)
        assert torch.equal(c.weight[a, h, b], torch.where(good, w0[page, h, place], torch.zeros((), device="cuda")))
    assert bad > 0
    assert torch.equal(c.k[:pages - new_cols], k0[:pages - new_cols]) and torch.equal(c.weight[:pages - new_cols], w0[:pages - new_cols])


def test_numbers_that_do_not_fit_are_refused():
    c = kv.PagedKV.allocate(8, PAGE, 1, 64, torch.float16, weight=True)
    x, table, n = torch.zeros(1, 1, 64, dtype=torch.float16, device="cuda"), to_int([[0]]), to_int([1])
    for bad in (dict(max_length=2 ** 40), dict(window=2 ** 33), dict(window=-2 ** 40), dict(window=0.5)):
        with pytest.raises(ValueError):
            c.attend(x, table, n, **bad)
    for bad in (dict(recent=2 ** 31), dict(first=-2 ** 31 - 1), dict(max_length=2 ** 40)):
        with pytest.raises(ValueError):
            c.evict(table, n, n, to_int([[1]]), **bad)
    with pytest.raises(FcsimError):                    # (infinity in 32 bits)
        c.attend(x, table, n, scale=1e300)
    with pytest.raises(FcsimError):
        c.append(x, x, x, None, torch.tensor([0], device="cuda"), eps=1e300)
    c.check()


# ------------------------------------------------------------------------------------------ calls
def test_layers_share_a_workspace_and_only_its_counters_are_cleared():
    """One workspace per stream whatever the number of caches; of a new one the part that has to be zero is cleared, no more."""
    g = gen(1)
    make = lambda: kv.PagedKV.allocate(600, PAGE, 2, 64, torch.float16, weight=True)  # noqa: E731
    a, b = make(), make()
    for c in (a, b):
        c.k.normal_(generator=g), c.v.normal_(generator=g)
    table = torch.arange(600, dtype=torch.int32, device="cuda").view(2, 300)
    q = torch.randn(2, 16, 64, generator=g, device="cuda").half()
    ln = to_int([4800, 4701])
    with torch.cuda.stream(torch.cuda.Stream()):
        old = torch.full((96 << 20,), 255, dtype=torch.uint8, device="cuda")   # what the allocator hands out next
        del old
        first = a.attend(q, table, ln, add_weight=True, return_lse=True)
        stream = torch.cuda.current_stream().cuda_stream
        work = a._workspaces[stream]
        assert b.attend(q, table, ln) is not None and b._workspaces[stream] is work
        assert not bool(work[:64 * 1024].any())
        torch.cuda.synchronize()
        before = a.weight.clone()
        a.weight.zero_()
        again = a.attend(q, table, ln, add_weight=True, return_lse=True)
        assert all(torch.equal(x, y) for x, y in zip(first, again)) and torch.equal(before, a.weight)
    # under capture: a call's own workspace, of which the graph clears the counters
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        out = a.attend(q, table, ln, return_lse=True)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0], first[0]) and torch.equal(out[1], first[1])


def test_a_fresh_workspace_is_not_cleared_whole():
    c = kv.PagedKV.allocate(64, PAGE, 2, 64, torch.float16)
    with torch.cuda.stream(torch.cuda.Stream()):
        size = 8 << 20
        old = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        del old
        buf = c._workspace(torch.cuda.current_stream().cuda_stream, size, 64 * 1024)
        assert buf.numel() >= size and not bool(buf[:64 * 1024].any()) and bool((buf[64 * 1024:size] == 255).all())
        assert c._workspace(0, 128, 0).numel() >= 128


def test_an_eviction_keeps_no_workspace():
    c = kv.PagedKV.allocate(8, PAGE, 1, 64, torch.float16, weight=True)
    with torch.cuda.stream(torch.cuda.Stream()):
        c.evict(to_int([[0, 1]]), to_int([32]), to_int([16]), to_int([[2]]))
        assert torch.cuda.current_stream().cuda_stream not in c._workspaces
    c.check()


def test_threads_with_caches_of_their_own_share_a_stream():
    import threading
    g = gen(2)
    stream, got, want = torch.cuda.Stream(), {}, {}
    caches = []
    for i in range(4):
        c = kv.PagedKV.allocate(300, PAGE, 2, 64, torch.float16, weight=True)
        c.k.normal_(generator=g), c.v.normal_(generator=g)
        table = torch.arange(300, dtype=torch.int32, device="cuda").view(3, 100)
        caches.append((c, torch.randn(3, 8, 64, generator=g, device="cuda").half(), table, to_int([1600, 1500 - i, 40 * i])))
    for i, (c, q, table, n) in enumerate(caches):
        want[i] = c.attend(q, table, n, add_weight=True), c.weight.clone()
        c.weight.zero_()
    torch.cuda.synchronize()

    def work(i):
        c, q, table, n = caches[i]
        with torch.cuda.stream(stream):
            for _ in range(50):
                c.weight.zero_()
                got[i] = c.attend(q, table, n, add_weight=True)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i, (c, *_) in enumerate(caches):
        assert torch.equal(got[i], want[i][0]) and torch.equal(c.weight, want[i][1])
        c.check()


def test_check_waits_for_calls_on_every_stream():
    c = kv.PagedKV.allocate(8, PAGE, 1, 64, torch.float16)
    q, table, n = torch.zeros(1, 1, 64, dtype=torch.float16, device="cuda"), to_int([[99]]), to_int([5])
    x = torch.randn(8192, 8192, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        for _ in range(10):
            x = x @ x                                   # long work before the call
        c.attend(q, table, n)
    with pytest.raises(ValueError, match="page"):
        c.check()
    torch.cuda.synchronize()
    c.check()


def test_a_cache_made_behind_long_work_is_ready_for_other_streams():
    k, v = (torch.zeros(8, PAGE, 1, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    q, table, n = torch.zeros(1, 1, 64, dtype=torch.float16, device="cuda"), to_int([[99]]), to_int([5])
    x = torch.randn(8192, 8192, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        for _ in range(10):
            x = x @ x
        c = kv.PagedKV(k, v)                            # its status word is cleared behind that
    with torch.cuda.stream(torch.cuda.Stream()):
        c.attend(q, table, n)
    torch.cuda.synchronize()
    with pytest.raises(ValueError, match="page"):
        c.check()


def test_tensors_that_want_a_gradient_are_refused():
    """There is no backward pass: results without one must not be taken for results with it."""
    c = kv.PagedKV.allocate(8, PAGE, 1, 64, torch.float16)
    x = torch.randn(1, 1, 64, device="cuda").half()
    slot, table, n = torch.tensor([0], device="cuda"), to_int([[0]]), to_int([1])
    w, rope = torch.ones(64, dtype=torch.float16, device="cuda"), torch.rand(4, 64, device="cuda")
    g = lambda t: t.detach().clone().requires_grad_()  # noqa: E731
    for bad in (dict(q=g(x)), dict(k=g(x)), dict(v=g(x)), dict(q_norm=g(w)), dict(k_norm=g(w)), dict(rope=g(rope))):
        args = {**dict(q=x, k=x, v=x, positions=to_int([0]), slots=slot, rope=rope, q_norm=w, k_norm=w), **bad}
        with pytest.raises(ValueError, match="gradient"):
            c.append(**args)
        with torch.no_grad():
            c.append(**args)
    with pytest.raises(ValueError, match="gradient"):
        c.attend(g(x), table, n)
    with torch.inference_mode():
        c.attend(x, table, n)
    with torch.no_grad():
        out = c.attend(g(x), table, n)
    assert not out.requires_grad
    c.check()


# ------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("scale", [1e-39, -1e-39, 1e-44, 2.0 ** -127])
def test_append_by_scales_whose_reciprocal_is_not_finite(scale):
    """What is stored is x / scale: zero stays zero, the rest reaches the type's end, or less where x is as small."""
    c = kv.PagedKV.allocate(2, PAGE, 1, 64, torch.float8_e4m3fn, k_scale=torch.tensor([scale], device="cuda"), v_scale=torch.tensor([scale], device="cuda"))
    x = torch.zeros(1, 1, 64, device="cuda")
    x[..., 0], x[..., 1], x[..., 2], x[..., 3] = 1.0, -1.0, scale, 2 * scale
    x = x.bfloat16()
    c.append(None, x, x, None, torch.tensor([3], device="cuda"))
    c.check()
    want = (x.double() / torch.tensor(scale, device="cuda").float().double()).clamp(-448, 448)[0, 0]
    for pool in (c.k, c.v):
        got = pool[0, 3, 0].float().double()
        assert bool(((got - want).abs() <= UNIT[torch.float8_e4m3fn] * want.abs()).all()), got[:4]
