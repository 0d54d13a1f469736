"""The paged cache's operators on the GPU against plain 64-bit forms of their definitions.

The bounds are those of kv_common: roundings to the stored types that the operators state, and 32-bit sums."""
import math

import pytest
import torch

from kv_common import DT, TINY, UNIT, assert_attend, make_pool, make_table, ref_append, ref_evict, wide
from paper_2604_11001_b200 import binding as fb
from paper_2604_11001_b200 import kvcache as kv

pytestmark = pytest.mark.gpu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def make_cache(g, n_pages, page, n_kv, head_dim, cache, heads_first=False, weight=True):
    scales = [0.25 + torch.rand(n_kv, generator=g, device="cuda") if cache == "e4m3" else None for _ in range(2)]
    w = torch.rand(n_pages, n_kv, page, generator=g, device="cuda") if weight else None
    return kv.PagedKV(make_pool(g, n_pages, page, n_kv, head_dim, cache, heads_first),
                      make_pool(g, n_pages, page, n_kv, head_dim, cache, heads_first), w, *scales)


# ------------------------------------------------------------------------------------------------- attend
def run_attend(seed, lengths, heads, n_kv, head_dim, page, dtype="bf16", cache="bf16", window=0, heads_first=False,
               add_weight=True, scale=None, spoil=True, cols=None):
    g = gen(seed)
    need = sum(-(-n // page) for n in lengths)
    c = make_cache(g, need + 3, page, n_kv, head_dim, cache, heads_first)
    table, _ = make_table(g, lengths, page, need + 3, cols=cols)
    if spoil:  # what no request holds must not be seen: NaN in every place that no token has, wild page numbers
        held = torch.zeros(need + 3, page, dtype=torch.bool)
        for r, n in enumerate(lengths):
            for i in range(-(-n // page)):
                held[int(table[r, i]), :min(page, n - i * page)] = True
        bad = ~held.cuda()
        for pool in (c.k, c.v):
            if pool.dtype == torch.float8_e4m3fn:
                pool.view(torch.uint8)[bad] = 0x7f
            else:
                pool[bad] = float("nan")
        table[table < 0] = 2 ** 31 - 1
    q = randn(g, len(lengths), heads, head_dim, dtype=DT[dtype])
    before = c.weight.clone()
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out, lse = c.attend(q, table, ln, window=window, add_weight=add_weight, return_lse=True, scale=scale)
    c.check()
    assert_attend(c, q, table, lengths, out, lse, before if add_weight else None, window=window, scale=scale)
    if not add_weight:
        assert torch.equal(before, c.weight)
    again = c.attend(q, table, ln, window=window, scale=scale)
    assert torch.equal(again, out)    # sums in a fixed order: the same bits on every call


EDGES = [0, 1, 2, 7, 8, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000]


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("head_dim", [16, 64, 80, 128, 192, 256])
def test_attend_widths_and_types(dtype, cache, head_dim):
    run_attend(head_dim, EDGES, 8, 2, head_dim, 16, dtype, cache)


@pytest.mark.parametrize("heads,n_kv", [(1, 1), (2, 1), (3, 3), (7, 1), (9, 1), (16, 1), (34, 2), (12, 4), (24, 1), (71, 1),
                                        (64, 8), (130, 2)])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_attend_head_groups(heads, n_kv, cache):
    run_attend(heads, [0, 1, 5, 70, 300, 1111], heads, n_kv, 64, 16, "bf16", cache)


@pytest.mark.parametrize("head_dim", [8, 24, 40, 120, 248])
def test_attend_narrow_and_odd_widths(head_dim):
    run_attend(head_dim, [3, 0, 129, 640], 6, 2, head_dim, 16, "f16", "f16")


@pytest.mark.parametrize("page", [1, 3, 5, 16, 48, 100, 128, 1024])
@pytest.mark.parametrize("heads_first", [False, True])
def test_attend_pages(page, heads_first):
    run_attend(page, [1, 2, 47, 48, 49, 700, 0, 2049], 8, 4, 64, page, heads_first=heads_first)


@pytest.mark.parametrize("window", [1, 15, 16, 64, 65, 1000, 5000])
@pytest.mark.parametrize("cache", ["f16", "e4m3"])
def test_attend_window(window, cache):
    run_attend(window, [0, 1, 16, 65, 66, 999, 1000, 1001, 3001], 4, 2, 128, 16, "f16", cache, window=window)


@pytest.mark.parametrize("lengths", [[20011], [1] * 700, [0] * 9, [0, 0, 5], [9000, 1, 0, 17, 8000, 3],
                                     [64 * i for i in range(40)], [16384]])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_attend_few_and_many_requests(lengths, cache):
    run_attend(len(lengths), lengths, 16, 2, 128, 16, "bf16", cache, spoil=len(lengths) < 100)


@pytest.mark.parametrize("scale", [0.0, 1.0, -0.3, 3.0])
def test_attend_scale(scale):
    run_attend(3, [5, 200, 777], 8, 2, 64, 16, "f16", "f16", scale=scale)


def test_attend_without_weights_and_wide_table():
    run_attend(4, [5, 200, 777], 8, 2, 64, 16, add_weight=False, cols=500)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_attend_strided_query_and_shared_pages(cache):
    """q as a slice of a packed projection, heads apart; several requests that read the same pages."""
    g = gen(11)
    c = make_cache(g, 20, 16, 2, 64, cache)
    x = randn(g, 5, 20 * 64, dtype=torch.bfloat16)
    q = x[:, 4 * 64:16 * 64].view(5, 6, 128)[:, :, :64]
    table = torch.arange(20, device="cuda", dtype=torch.int32).repeat(5, 2)[:, :20]
    lengths = [300, 17, 1, 320, 299]
    out, lse = c.attend(q, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), return_lse=True)
    assert_attend(c, q, table, lengths, out, lse)


@pytest.mark.parametrize("cache,big", [("bf16", 3e38), ("f16", 60000.0), ("e4m3", 448.0)])
def test_attend_extreme_logits(cache, big):
    """One key far above the rest takes everything; keys at the type's ends elsewhere give the lowest logits, which
    must neither overflow the running maximum nor lose the sum."""
    g = gen(5)
    dtype = "bf16" if cache == "bf16" else "f16"
    c = make_cache(g, 40, 16, 1, 64, cache, weight=False)
    table = torch.arange(40, device="cuda", dtype=torch.int32)[None]
    q = torch.zeros(1, 4, 64, dtype=DT[dtype], device="cuda")
    q[..., 0] = 1.0
    for pool, val in ((c.k, -big),):
        pool.view(torch.uint8).zero_() if cache == "e4m3" else pool.zero_()
        col = torch.full((40, 16, 1), val, device="cuda").to(DT[cache])
        if cache == "e4m3":
            pool.view(torch.uint8)[..., 0] = col.view(torch.uint8)
            pool.view(torch.uint8)[7, 3, 0, 0] = torch.tensor([big], device="cuda").to(DT[cache]).view(torch.uint8)[0]
        else:
            pool[..., 0] = col
            pool[7, 3, 0, 0] = big
    out, lse = c.attend(q, table, torch.tensor([640], dtype=torch.int32, device="cuda"), return_lse=True, scale=1.0)
    want = wide(c.v[7, 3, 0]) * (c.v_scale.double() if cache == "e4m3" else 1.0)
    assert bool(((wide(out[0]) - want).abs() <= UNIT[q.dtype] * 2 * want.abs() + TINY[q.dtype]).all())
    # without that key all logits are the same lowest value: the plain mean, and a finite log-sum-exp
    n = 7 * 16
    out, lse = c.attend(q, table, torch.tensor([n], dtype=torch.int32, device="cuda"), return_lse=True, scale=1.0)
    v = wide(c.v[:7]).reshape(n, 64) * (c.v_scale.double() if cache == "e4m3" else 1.0)
    tol = UNIT[q.dtype] * (v.mean(0).abs() + v.abs().mean(0)) + 2.0 ** -12 * v.abs().mean(0) + TINY[q.dtype]
    assert bool(((wide(out[0]) - v.mean(0)).abs() <= tol).all())
    assert bool(torch.isfinite(lse).all())


def test_attend_infinite_and_nan_values_stay_with_their_request():
    g = gen(6)
    c = make_cache(g, 64, 16, 2, 64, "f16")
    table = torch.arange(64, device="cuda", dtype=torch.int32).view(4, 16)
    lengths = [200, 130, 256, 70]
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q = randn(g, 4, 4, 64, dtype=torch.float16)
    clean, _ = c.attend(q, table, ln, return_lse=True)
    c.k[int(table[1, 2]), 3] = float("nan")
    c.k[int(table[2, 0]), 1, 0] = float("-inf")   # q has both signs: -inf and inf logits, or NaN from inf - inf
    c.v[int(table[3, 1]), 2, 1, 5] = float("inf")
    out, lse = c.attend(q, table, ln, return_lse=True)
    assert torch.equal(out[0], clean[0])
    assert bool(torch.isnan(out[1]).all()) and bool(torch.isnan(lse[1]).all())
    assert torch.equal(out[2, 2:], clean[2, 2:])                      # the other kv head's query heads
    assert bool((out[3, 2:, 5] == float("inf")).all())
    keep = [i for i in range(64) if i != 5]
    assert torch.equal(out[3, 2:, keep], clean[3, 2:, keep]) and torch.equal(out[3, :2], clean[3, :2])


def test_attend_minus_infinity_logits_count_as_nothing():
    c = make_cache(gen(8), 8, 16, 1, 64, "bf16", weight=False)
    table = torch.arange(8, device="cuda", dtype=torch.int32)[None]
    q = torch.ones(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    c.k[...] = 0
    c.k[:5] = float("-inf")                                          # the first 80 tokens, whole tiles among them
    out, lse = c.attend(q, table, torch.tensor([128], dtype=torch.int32, device="cuda"), return_lse=True)
    v = wide(c.v[5:]).reshape(48, 64)
    tol = UNIT[q.dtype] * (v.mean(0).abs() + v.abs().mean(0)) + 2.0 ** -14 * v.abs().mean(0)
    assert bool(((wide(out[0]) - v.mean(0)).abs() <= tol).all())
    assert bool(((lse - math.log(48)).abs() < 1e-5).all())
    out, lse = c.attend(q, table, torch.tensor([80], dtype=torch.int32, device="cuda"), return_lse=True)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())   # nothing left: as without tokens


def test_attend_calls_of_different_shapes_share_a_workspace():
    """One cache, one stream: calls whose grids, parts and joins differ, each after another kind."""
    g = gen(17)
    c = make_cache(g, 2000, 16, 4, 64, "bf16")
    kinds = [([9000], 16), ([40] * 300, 4), ([700] * 20, 32), ([1], 4), ([16000], 4), ([300, 5, 2000], 64), ([18] * 900, 16), ([4000] * 4, 8)]
    for turn in range(3):
        for lengths, heads in kinds[turn:] + kinds[:turn]:
            table, _ = make_table(g, lengths, 16, 2000)
            q = randn(g, len(lengths), heads, 64, dtype=torch.bfloat16)
            before = c.weight.clone()
            add = (turn + heads) % 3 == 0
            out, lse = c.attend(q, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), add_weight=add, return_lse=True)
            assert_attend(c, q, table, lengths, out, lse, before if add else None)
    zeroed = next(iter(c._workspaces.values()))[:64 * 1024]
    assert not bool(zeroed.any())
    c.check()


def test_append_and_evict_in_a_graph():
    g = gen(18)
    c = make_cache(g, 64, 16, 2, 64, "bf16")
    to_int = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table, new = to_int([list(range(20)), list(range(20, 40))]), to_int([[40, 41, 42, 43], [44, 45, 46, 47]])
    lengths, budget = to_int([300, 77]), to_int([50, 64])
    x = randn(g, 2, 2, 64, dtype=torch.bfloat16)
    slots = torch.tensor([5, 20 * 16 + 3], device="cuda")
    want_n, want_kept = c.evict(table, lengths, budget, new, recent=5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        q = c.append(x, x, x, None, slots)
        n, kept = c.evict(table, lengths, budget, new, recent=5)
    c.weight.copy_(torch.rand(c.weight.shape, generator=g, device="cuda") + 1)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(q, x) and torch.equal(c.k[0, 5], x[0]) and torch.equal(n, want_n)
    weight = c.weight.clone()
    weight[0, :, 5] = 0        # the appended tokens have no weight yet
    for r, (length, b) in enumerate(((300, 50), (77, 64))):
        t = torch.arange(length, device="cuda")
        w = weight[table[r].long()[t // 16], :, t % 16].cpu()
        for h in range(2):
            assert kept[r, h, :b].tolist() == ref_evict(w[:, h].tolist(), length, b, 5, 0)
    c.check()


def test_attend_beyond_32_bit_offsets():
    """A pool of more than 2^32 elements: the pages that a request holds lie at its two ends."""
    page, n_kv, D = 16, 8, 128
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
    q = randn(g, 2, 16, D, dtype=torch.bfloat16)
    lengths = [77, 80]
    out, lse = c.attend(q, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), return_lse=True)
    assert_attend(c, q, table, lengths, out, lse)
    slots = torch.tensor([n_pages * page - 1, 5], dtype=torch.int64, device="cuda")
    x = randn(g, 2, n_kv, D, dtype=torch.bfloat16)
    c.append(None, x, x, None, slots)
    assert torch.equal(c.k[n_pages - 1, page - 1], x[0]) and torch.equal(c.v[0, 5], x[1])
    c.check()


def test_attend_bad_pages_and_lengths_are_flagged():
    g = gen(12)
    c = make_cache(g, 8, 16, 2, 64, "bf16")
    table = torch.arange(8, device="cuda", dtype=torch.int32).view(2, 4)
    q = randn(g, 2, 4, 64, dtype=torch.bfloat16)
    ok, ok_lse = c.attend(q, table, torch.tensor([64, 64], dtype=torch.int32, device="cuda"), return_lse=True)
    c.check()
    for wild in (-1, 8, 2 ** 31 - 1, -2 ** 31):
        t = table.clone()
        t[0, 1] = wild
        out, lse = c.attend(q, t, torch.tensor([64, 64], dtype=torch.int32, device="cuda"), return_lse=True)
        assert torch.equal(out[1], ok[1])
        # the tokens of the bad page are left out
        skip = t.clone()
        skip[0, 1:3] = t[0, 2:4]
        assert_attend(c, q, skip, [48, 64], out, lse)
        with pytest.raises(ValueError, match="page"):
            c.check()
    before = c.weight.clone()
    t = table.clone()
    t[0, 0] = 99
    c.attend(q, t, torch.tensor([16, 0], dtype=torch.int32, device="cuda"), add_weight=True)
    assert torch.equal(before, c.weight)
    with pytest.raises(ValueError, match="page"):
        c.check()
    out, lse = c.attend(q, table, torch.tensor([-5, 65], dtype=torch.int32, device="cuda"), return_lse=True)
    assert bool((out[0] == 0).all()) and torch.equal(out[1], ok[1])
    with pytest.raises(ValueError, match="length"):
        c.check()
    c.check()


def test_attend_on_streams_and_in_a_graph():
    g = gen(13)
    c = make_cache(g, 400, 16, 2, 64, "bf16")
    lengths = [3000, 1, 700]
    table, _ = make_table(g, lengths, 16, 400)
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q = randn(g, 3, 16, 64, dtype=torch.bfloat16)
    want = c.attend(q, table, ln)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for i in range(30):
        with torch.cuda.stream(streams[i % 3]):
            got.append(c.attend(q, table, ln))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        out = c.attend(q, table, ln, add_weight=True)
    before = c.weight.clone()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    one = c.weight.clone()
    c.weight.copy_(before)
    for _ in range(2):
        c.attend(q, table, ln, add_weight=True)
    assert torch.equal(one, c.weight)


# ------------------------------------------------------------------------------------------------- append
def run_append(seed, n, heads, n_kv, head_dim, page, dtype="bf16", cache="bf16", rope_dim=None, interleaved=False,
               norm=True, heads_first=False, packed=True, eps=1e-6):
    g = gen(seed)
    n_pages = -(-n // page) + 3
    c = make_cache(g, n_pages, page, n_kv, head_dim, cache, heads_first)
    if packed:
        x = 3 * randn(g, n, (heads + 2 * n_kv) * head_dim, dtype=DT[dtype])
        cut = [heads * head_dim, (heads + n_kv) * head_dim]
        q, k, v = (y.view(n, -1, head_dim) for y in (x[:, :cut[0]], x[:, cut[0]:cut[1]], x[:, cut[1]:]))
    else:  # [heads, tokens, head_dim] in memory
        q, k, v = (3 * randn(g, h, n, head_dim, dtype=DT[dtype]).transpose(0, 1) for h in (heads, n_kv, n_kv))
    w = [1 + 0.2 * randn(g, head_dim, dtype=DT[dtype]) if norm else None for _ in range(2)]
    rope = positions = None
    if rope_dim:
        rope = torch.empty(501, rope_dim, device="cuda").uniform_(-1, 1, generator=g)
        positions = torch.randint(0, 501, (n,), generator=g, device="cuda", dtype=torch.int32)
    slots = torch.randperm(n_pages * page, generator=g, device="cuda")[:n].to(torch.int64)
    slots[::7] = -1
    kc, vc, wc = c.k.clone(), c.v.clone(), c.weight.clone()
    out = c.append(q, k, v, positions, slots, rope=rope, interleaved=interleaved, q_norm=w[0], k_norm=w[1], eps=eps)
    c.check()
    # 32-bit sums of D squares, a square root, a division, three products: 2^-18 of the row is far above their
    # errors for D <= 256 (256 * 2^-24 / 2 = 2^-17 / 2 at the very worst); then one rounding
    for got, (x, wn) in ((out, (q, w[0])),):
        ref, size = ref_append(x, wn, rope, positions, interleaved, eps)
        tol = UNIT[out.dtype] * ref.abs() + 2.0 ** -17 * size + TINY[out.dtype]
        assert bool(((wide(got) - ref).abs() <= tol).all())
    held = slots >= 0
    pg, pl = slots[held] // page, slots[held] % page
    refk, size = ref_append(k, w[1], rope, positions, interleaved, eps)
    refv = wide(v)
    if c.k_scale is not None:
        refk, size = refk / c.k_scale.double()[:, None], size / c.k_scale.double()[:, None]
        refv = refv / c.v_scale.double()[:, None]
        refk, refv = refk.clamp(-448, 448), refv.clamp(-448, 448)
    gotk, gotv = wide(c.k)[pg, pl], wide(c.v)[pg, pl]
    tol = UNIT[DT[cache]] * refk.abs() + 2.0 ** -17 * size + TINY[DT[cache]]
    assert bool(((gotk - refk[held]).abs() <= tol[held]).all())
    if c.k_scale is None:
        assert torch.equal(gotv, refv[held])
    else:
        tol = UNIT[DT[cache]] * (1 + 2.0 ** -20) * refv.abs() + TINY[DT[cache]]
        assert bool(((gotv - refv[held]).abs() <= tol[held]).all())
    # nothing else moved
    mark = torch.zeros(n_pages, page, dtype=torch.bool, device="cuda")
    mark[pg, pl] = True
    byte = torch.uint8 if cache == "e4m3" else torch.int16
    assert torch.equal(c.k.view(byte)[~mark], kc.view(byte)[~mark]) and torch.equal(c.v.view(byte)[~mark], vc.view(byte)[~mark])
    wt, wct = c.weight.transpose(1, 2), wc.transpose(1, 2)
    assert bool((wt[mark] == 0).all()) and torch.equal(wt[~mark], wct[~mark])


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("head_dim,rope_dim,interleaved", [(64, 64, False), (128, 64, False), (128, 128, True),
                                                           (96, 96, False), (80, 32, True), (256, 256, False),
                                                           (112, 112, False), (16, 16, False), (192, 0, False),
                                                           (128, 6, True)])
def test_append_types_and_widths(dtype, cache, head_dim, rope_dim, interleaved):
    run_append(head_dim + rope_dim, 37, 6, 2, head_dim, 16, dtype, cache, rope_dim, interleaved)


@pytest.mark.parametrize("n", [1, 2, 3, 255, 1025])
@pytest.mark.parametrize("heads,n_kv", [(1, 1), (5, 1), (64, 8), (6, 3)])
def test_append_counts(n, heads, n_kv):
    run_append(n + heads, n, heads, n_kv, 64, 5, rope_dim=64)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("head_dim", [8, 24, 40, 72, 248])
def test_append_odd_widths(norm, head_dim):
    run_append(head_dim, 33, 3, 1, head_dim, 16, "f16", "f16", rope_dim=head_dim // 16 * 16, norm=norm)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_append_heads_outermost(cache):
    run_append(1, 70, 8, 4, 128, 16, "bf16", cache, 128, heads_first=True, packed=False)


def test_append_nothing_and_without_queries():
    g = gen(3)
    c = make_cache(g, 4, 16, 2, 64, "bf16")
    empty = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    out = c.append(empty, empty, empty, None, torch.empty(0, dtype=torch.int64, device="cuda"))
    assert tuple(out.shape) == (0, 2, 64)
    x = randn(g, 3, 2, 64, dtype=torch.bfloat16)
    assert c.append(None, x, x, None, torch.tensor([1, 17, 63], device="cuda")) is None
    assert torch.equal(c.k[1, 1], x[1]) and torch.equal(c.v[3, 15], x[2])
    c.check()


def test_append_zero_rows_large_values_and_saturation():
    """A zero row stays zero under the norm (eps > 0); f16's largest values do not overflow the 32-bit sum of squares;
    e4m3 takes +-448 beyond its range and keeps NaN."""
    c = make_cache(gen(4), 2, 16, 1, 64, "f16")
    x = torch.zeros(2, 1, 64, dtype=torch.float16, device="cuda")
    x[1] = 65504
    w = torch.ones(64, dtype=torch.float16, device="cuda")
    out = c.append(x, x, x, None, torch.tensor([0, 1], device="cuda"), q_norm=w, k_norm=w)
    assert bool((out[0] == 0).all()) and bool((out[1] == 1).all()) and bool((c.k[0, 1] == 1).all())
    c = make_cache(gen(4), 2, 16, 1, 64, "e4m3")
    y = torch.zeros(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    y[..., 0], y[..., 1], y[..., 2], y[..., 3], y[..., 4] = 1e30, -1e30, float("inf"), float("nan"), 1e-30
    c.append(None, y, y, None, torch.tensor([3], device="cuda"))
    got = c.v[0, 3, 0].float().tolist()[:5]
    assert got[0] == 448 and got[1] == -448 and got[2] == 448 and math.isnan(got[3]) and got[4] == 0


def test_append_bad_slots_and_positions_are_flagged():
    g = gen(5)
    c = make_cache(g, 2, 16, 2, 64, "bf16")
    x = randn(g, 4, 2, 64, dtype=torch.bfloat16)
    k0, v0, w0 = c.k.clone(), c.v.clone(), c.weight.clone()
    rope = torch.rand(10, 64, generator=g, device="cuda")
    pos = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
    slots = torch.tensor([32, 2 ** 31, 2 ** 40, 2 ** 62], device="cuda")
    ref = c.append(x, x, x, pos, torch.full((4,), -1, device="cuda"), rope=rope)
    c.check()
    out = c.append(x, x, x, pos, slots, rope=rope)
    assert torch.equal(out, ref)
    with pytest.raises(ValueError, match="slot"):
        c.check()
    pos = torch.tensor([0, 10, -1, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    out = c.append(x, x, x, pos, torch.tensor([-1, 1, 2, 3], device="cuda"), rope=rope)
    assert torch.equal(out[0], ref[0]) and bool((out[1:] == 0).all())
    with pytest.raises(ValueError, match="position"):
        c.check()
    assert torch.equal(c.k, k0) and torch.equal(c.v, v0) and torch.equal(c.weight, w0)


# ------------------------------------------------------------------------------------------------- evict
def run_evict(seed, lengths, budgets, recent, first, n_kv=2, head_dim=64, page=16, cache="bf16", heads_first=False,
              values="spread", max_budget=None):
    g = gen(seed)
    top = max(budgets + [1]) if max_budget is None else max_budget
    old = sum(-(-n // page) for n in lengths)
    n_pages = old + len(lengths) * (-(-top // page)) + 3
    c = make_cache(g, n_pages, page, n_kv, head_dim, cache, heads_first)
    if values == "spread":
        c.weight.copy_(torch.exp(2 * randn(g, *c.weight.shape)) * (torch.rand(c.weight.shape, generator=g, device="cuda") > 0.1))
    elif values == "ties":
        c.weight.copy_(torch.randint(0, 3, c.weight.shape, generator=g, device="cuda").float())
    elif values == "same":
        c.weight.fill_(0.0)
    else:
        pick = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 1e-45, -1e-45, 3e38, -3e38, 1.0], device="cuda")
        c.weight.copy_(pick[torch.randint(0, 10, c.weight.shape, generator=g, device="cuda")])
    table, left = make_table(g, lengths, page, n_pages, fill=2 ** 31 - 1)
    new_cols = max(1, -(-top // page))
    new_table = torch.tensor(left[:len(lengths) * new_cols], dtype=torch.int32, device="cuda").view(len(lengths), new_cols)
    k0, v0, w0 = c.k.clone(), c.v.clone(), c.weight.clone()
    to_int = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    new_lengths, kept = c.evict(table, to_int(lengths), to_int(budgets), new_table, recent=recent, first=first, max_budget=top)
    c.check()
    assert tuple(kept.shape) == (len(lengths), n_kv, top)
    byte = torch.uint8 if cache == "e4m3" else torch.int16
    wantk, wantv, wantw = k0.clone().view(byte), v0.clone().view(byte), w0.clone()
    kb, vb = k0.view(byte), v0.view(byte)
    for r, n in enumerate(lengths):
        keep = min(n, budgets[r])
        assert int(new_lengths[r]) == keep
        t = torch.arange(n, device="cuda")
        pg, pl = table[r].long()[t // page], t % page
        w = w0[pg, :, pl].cpu()
        for h in range(n_kv):
            want = ref_evict(w[:, h].tolist(), n, budgets[r], recent, first)
            assert kept[r, h, :keep].tolist() == want, (r, h)
            assert bool((kept[r, h, keep:] == -1).all())
            src = torch.tensor(want, dtype=torch.long, device="cuda")
            dst = torch.arange(keep, device="cuda")
            a, b = new_table[r].long()[dst // page], dst % page
            wantk[a, b, h] = kb[pg[src], pl[src], h]
            wantv[a, b, h] = vb[pg[src], pl[src], h]
            wantw[a, h, b] = w0[pg[src], h, pl[src]]
    assert torch.equal(c.k.view(byte), wantk) and torch.equal(c.v.view(byte), wantv)
    assert torch.equal(c.weight.view(torch.int32), wantw.view(torch.int32))


@pytest.mark.parametrize("values", ["spread", "ties", "same", "odd"])
@pytest.mark.parametrize("recent,first", [(0, 0), (8, 0), (0, 4), (13, 3), (500, 500)])
def test_evict_rules(values, recent, first):
    lengths = [0, 1, 2, 15, 16, 17, 64, 100, 257, 1000]
    run_evict(recent + first, lengths, [0, 1, 1, 10, 16, 16, 33, 100, 64, 200], recent, first, values=values)


@pytest.mark.parametrize("cache", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("head_dim", [16, 64, 96, 128, 256])
@pytest.mark.parametrize("heads_first", [False, True])
def test_evict_types_and_widths(cache, head_dim, heads_first):
    run_evict(head_dim, [90, 300, 5], [40, 100, 40], 10, 2, 3, head_dim, 16, cache, heads_first)


@pytest.mark.parametrize("page", [1, 3, 5, 48, 128])
def test_evict_pages(page):
    run_evict(page, [47, 48, 49, 700], [10, 48, 30, 129], 5, 1, 2, 64, page)


@pytest.mark.parametrize("lengths,budgets", [([20000], [1]), ([20000], [19999]), ([33000, 70], [4096, 64]), ([70000], [700]),
                                             ([12, 5], [0, 0]), ([131072], [9000]), ([300] * 200, [100] * 200)])
@pytest.mark.parametrize("values", ["spread", "ties"])
def test_evict_sizes(lengths, budgets, values):
    run_evict(len(lengths), lengths, budgets, 0 if budgets[0] < 2 else 33, 0, 1 if lengths[0] > 300 else 2, 16, 16, values=values)


def test_evict_more_keys_than_shared_memory_holds():
    """Eight CTAs hold 393 216 keys; beyond that the weights are read again for every digit."""
    run_evict(9, [450001], [5000], 100, 3, 1, 16, 16)


def test_evict_wider_output_than_any_budget():
    run_evict(1, [40, 70], [16, 70], 4, 1, max_budget=300)


def test_evict_bad_values_are_flagged():
    g = gen(2)
    c = make_cache(g, 12, 16, 1, 64, "bf16")
    to_int = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table, new = to_int([[0, 1], [2, 3]]), to_int([[4], [5]])
    n, kept = c.evict(table, to_int([-3, 99]), to_int([5, 16]), new)
    assert n.tolist() == [0, 16]
    with pytest.raises(ValueError, match="length"):
        c.check()
    n, kept = c.evict(table, to_int([32, 32]), to_int([-1, 17]), new)
    assert n.tolist() == [0, 16]
    with pytest.raises(ValueError, match="budget"):
        c.check()
    # pages outside the pool: nothing is read or written there, the other request is served
    k0 = c.k.clone()
    n, kept = c.evict(to_int([[0, 77], [2, 3]]), to_int([32, 32]), to_int([8, 8]), to_int([[-9], [5]]))
    with pytest.raises(ValueError, match="page"):
        c.check()
    assert torch.equal(c.k[:5], k0[:5]) and torch.equal(c.k[6:], k0[6:])
    assert torch.equal(c.k[5, :8, 0], c.k[table[1].long()[kept[1, 0, :8].long() // 16], kept[1, 0, :8].long() % 16, 0])


# ------------------------------------------------------------------------------------------------- together
def test_slots_of_append_attend_evict():
    """A few requests grow token by token, are cut to a budget and go on, against the same steps in 64 bits."""
    g = gen(21)
    page, n_kv, heads, D, budget = 16, 2, 8, 64, 40
    c = make_cache(g, 64, page, n_kv, D, "f16")
    free = list(range(64))
    lengths = [30, 1, 17]
    tables = [[free.pop() for _ in range(5)] for _ in lengths]
    to_int = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    slot = lambda r, t: tables[r][t // page] * page + t % page  # noqa: E731
    prompt = randn(g, sum(lengths), n_kv, D, dtype=torch.float16)
    c.append(None, prompt, prompt, None, torch.tensor([slot(r, t) for r, n in enumerate(lengths) for t in range(n)], device="cuda"))
    for step in range(40):
        q, k, v = (randn(g, 3, h, D, dtype=torch.float16) for h in (heads, n_kv, n_kv))
        q = c.append(q, k, v, None, torch.tensor([slot(r, n) for r, n in enumerate(lengths)], device="cuda"))
        lengths = [n + 1 for n in lengths]
        before = c.weight.clone()
        table = to_int(tables)
        out, lse = c.attend(q, table, to_int(lengths), add_weight=True, return_lse=True)
        assert_attend(c, q, table, lengths, out, lse, before)
        for r in range(3):
            if lengths[r] > budget + 8:
                fresh = [free.pop() for _ in range(5)]
                n, kept = c.evict(table[r:r + 1], to_int([lengths[r]]), to_int([budget]), to_int([fresh]), recent=8, first=2)
                assert n.tolist() == [budget] and kept[0, 0, :2].tolist() == [0, 1]
                free += tables[r]
                tables[r], lengths[r] = fresh, budget
    c.check()


def test_a_call_on_the_wrong_device_or_type_is_refused():
    c = make_cache(gen(1), 4, 16, 2, 64, "bf16")
    q = torch.zeros(1, 4, 64, dtype=torch.float16, device="cuda")
    table, n = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    with pytest.raises(fb.FcsimError) as e:
        c.attend(q, table, n)                 # f16 queries over a bf16 cache
    assert e.value.code == -1
    q = q.bfloat16()
    for bad in (dict(q=q.cpu()), dict(q=q[:, :3]), dict(q=q[..., :32]), dict(table=table.long()), dict(lengths=n.long()),
                dict(lengths=n.cpu()), dict(max_length=17), dict(window=-1), dict(q=q.float()), dict(table=table[0])):
        with pytest.raises((ValueError, fb.FcsimError)):
            c.attend(**{**dict(q=q, table=table, lengths=n), **bad})


@pytest.mark.parametrize("cache,head_dim,heads,n_kv", [("bf16", 128, 64, 8), ("f16", 64, 16, 8), ("e4m3", 128, 64, 8), ("e4m3", 64, 24, 2),
                                                       ("bf16", 192, 48, 8), ("f16", 112, 96, 8)])
@pytest.mark.parametrize("window", [0, 37])
def test_attend_many_short_requests_and_a_few_long_ones(cache, head_dim, heads, n_kv, window):
    """More groups than warps on the GPU, most of one or two tiles, some cut among many."""
    import random
    rng = random.Random(head_dim + window)
    lengths = [rng.randint(0, 90) for _ in range(500)] + [2500, 1] + [rng.randint(100, 400) for _ in range(60)] + [0, 1300]
    run_attend(head_dim, lengths, heads, n_kv, head_dim, 16, "f16" if cache == "f16" else "bf16", cache, window=window, spoil=window > 0)


@pytest.mark.parametrize("requests,n_kv", [(1, 8), (3, 2), (37, 8), (220, 1), (300, 2)])
@pytest.mark.parametrize("length", [1, 64, 65, 300, 1024, 1025])
def test_attend_equal_lengths(requests, n_kv, length):
    """Every way of dividing the work: pieces of groups, whole groups, shares of units, warps alone."""
    run_attend(requests + length, [length] * requests, 4 * n_kv, n_kv, 64, 16, spoil=False)


@pytest.mark.parametrize("requests", [27, 28, 36, 37, 38, 55, 56, 74, 75, 160])
@pytest.mark.parametrize("longest", [64, 256, 257, 1100])
def test_attend_about_as_many_groups_as_workers(requests, longest):
    """One group more or less than the GPU holds CTAs or warps, all short or one among them long."""
    import random
    rng = random.Random(requests * longest)
    lengths = [rng.randint(0, min(longest, 256)) for _ in range(requests)]
    lengths[requests // 2] = longest
    run_attend(requests + longest, lengths, 16, 8, 128, 16, spoil=False)


@pytest.mark.parametrize("preset,cache,budget", [(1, "bf16", None), (1, "e4m3", 48), (6, "f16", 32)])
def test_slots_of_a_preset_in_seconds(preset, cache, budget):
    from paper_2604_11001_b200 import slot_time as st
    got = st.run(preset, slots=300, replicas=4, points=3, grow=80 if budget else 3, budget=budget, heads=8, kv_heads=2, head_dim=64, cache=cache)
    assert len(got["rows"]) >= 2 and all(r["us"] > 0 for r in got["rows"])
    if budget:
        assert all(r["longest"] <= budget for r in got["rows"])
    for g in got["groups"]:
        assert g["slot_us"] > 0 and math.isfinite(g["mean_latency_ms"]) and g["tokens_per_second"] > 0


def test_a_layer_grows_as_its_parts_do():
    """The example's slots against the same steps in 64 bits: lengths, places and the last slot's attention."""
    from paper_2604_11001_b200 import slot_time as st
    layer = st.Layer([5, 33, 16], heads=4, kv_heads=2, head_dim=64, cache="f16", budget=40, seed=3)
    for i in range(90):
        before = layer.cache.weight.clone()
        layer.grow()
    assert layer.positions.tolist() == [95, 123, 106]
    assert all(40 <= n < 40 + st.SLACK for n in layer.lengths.tolist())
    lengths = layer.lengths.tolist()
    q = randn(gen(1), 3, 4, 64, dtype=torch.float16)
    before = layer.cache.weight.clone()
    out, lse = layer.cache.attend(q, layer.table, layer.lengths, add_weight=True, return_lse=True)
    assert_attend(layer.cache, q, layer.table, lengths, out, lse, before)
    layer.cache.check()
