"""prefill against plain 64-bit forms of its definition: several query tokens per request over a paged cache."""
import math

import pytest
import torch

from kv_common import DT, make_table
from kv_prompt_common import assert_prompt
from test_kv_gpu import gen, make_cache, randn


def spoil(c, table, lengths, page, window, first, new):
    """What no row sees must not matter: NaN in every place without a token, wild page numbers behind the last and in between."""
    held = torch.zeros(c.n_pages, page, dtype=torch.bool)
    for r, n in enumerate(lengths):
        for i in range(-(-n // page)):
            if window and i * page >= first and (i + 1) * page <= n - new[r] - window + 1:
                table[r, i] = 2 ** 31 - 1
            else:
                held[int(table[r, i]), :min(page, n - i * page)] = True
    bad = ~held.cuda()
    for pool in (c.k, c.v):
        if pool.dtype == torch.float8_e4m3fn:
            pool.view(torch.uint8)[bad] = 0x7f
        else:
            pool[bad] = float("nan")
    table[table < 0] = 2 ** 31 - 1


def run_prefill(seed, new, lengths, heads, n_kv, head_dim, page, dtype="bf16", cache="bf16", window=0, first=0, heads_first=False,
                scale=None, max_length=None, spare_rows=(0, 0), again=True):
    g = gen(seed)
    need = sum(-(-n // page) for n in lengths)
    c = make_cache(g, need + 3, page, n_kv, head_dim, cache, heads_first)
    table, _ = make_table(g, lengths, page, need + 3)
    spoil(c, table, lengths, page, window, first, new)
    starts = [spare_rows[0]]
    for n in new:
        starts.append(starts[-1] + n)
    q = randn(g, starts[-1] + spare_rows[1], heads, head_dim, dtype=DT[dtype])
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    st = torch.tensor(starts, dtype=torch.int32, device="cuda")
    args = dict(window=window, first=first, scale=scale, max_length=max_length)
    out, lse = c.prefill(q, st, table, ln, return_lse=True, **args)
    c.check()
    args.pop("max_length")
    assert_prompt(c, q, starts, table, lengths, out, lse, **args)
    if again:
        assert torch.equal(c.prefill(q, st, table, ln, **args), out)    # sums in a fixed order: the same bits on every call
    return c, q, st, table, ln, out, lse


@pytest.mark.gpu
@pytest.mark.parametrize("new,length", [(1, 1), (2, 2), (5, 5), (16, 16), (17, 17), (32, 32), (33, 40), (64, 64), (100, 128), (128, 129), (129, 300), (300, 1000)])
def test_one_request(new, length):
    run_prefill(new, [new], [length], 8, 1, 128, 16)


NEW = [0, 1, 2, 7, 0, 16, 33, 65, 128, 200, 1]
LENGTHS = [5, 1, 2, 300, 0, 16, 40, 65, 513, 200, 777]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("head_dim", [16, 64, 80, 128, 192, 256])
def test_widths_and_types(dtype, cache, head_dim):
    run_prefill(head_dim, NEW, LENGTHS, 8, 2, head_dim, 16, dtype, cache)


@pytest.mark.gpu
@pytest.mark.parametrize("head_dim", [8, 24, 40, 72, 120, 136, 248])
def test_narrow_and_odd_widths(head_dim):
    run_prefill(head_dim, NEW, LENGTHS, 6, 2, head_dim, 16, "f16", "f16")


@pytest.mark.gpu
@pytest.mark.parametrize("heads,n_kv", [(1, 1), (3, 3), (7, 1), (9, 1), (16, 2), (34, 2), (24, 1), (71, 1), (64, 8), (130, 1), (300, 1), (520, 2)])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_head_groups(heads, n_kv, cache):
    run_prefill(heads, [3, 0, 40, 1, 70], [5, 9, 40, 300, 711], heads, n_kv, 64, 16, "bf16", cache)


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [130, 300])
def test_large_groups_of_wide_heads(heads):
    run_prefill(heads, [3, 20, 1], [5, 40, 300], heads, 1, 256, 16)


@pytest.mark.gpu
@pytest.mark.parametrize("page", [1, 3, 16, 24, 100, 128, 1024])
@pytest.mark.parametrize("heads_first", [False, True])
def test_pages(page, heads_first):
    run_prefill(page, [4, 1, 47, 100, 0, 200], [4, 129, 47, 700, 0, 2049], 8, 4, 64, page, heads_first=heads_first)


@pytest.mark.gpu
@pytest.mark.parametrize("window,first", [(1, 0), (1, 1), (15, 0), (64, 4), (100, 130), (128, 128), (300, 3), (1000, 64), (1, 700), (5000, 9)])
@pytest.mark.parametrize("cache,head_dim", [("f16", 128), ("e4m3", 64), ("f16", 256)])
def test_windows_and_first_tokens(window, first, cache, head_dim):
    run_prefill(window, [1, 16, 66, 300, 128, 50], [1, 16, 666, 1000, 128, 2000], 4, 2, head_dim, 16, "f16", cache, window=window, first=first)


@pytest.mark.gpu
@pytest.mark.parametrize("new,lengths", [([5], [20011]), ([1] * 300, [1] * 300), ([2000, 1, 0, 17], [9000, 1, 0, 8000]), ([1, 1], [30000, 5]),
                                         ([64 * (i % 3) for i in range(40)], [64 * i + 128 for i in range(40)]), ([0] * 9, [0, 3] * 4 + [1]), ([4096], [4096])])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_few_and_many_requests(new, lengths, cache):
    run_prefill(len(new), new, lengths, 16, 2, 128, 16, "bf16", cache)


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.0, 1.0, -0.3, 3.0])
@pytest.mark.parametrize("head_dim", [64, 256])
def test_scale(scale, head_dim):
    run_prefill(3, [5, 100, 200], [5, 200, 777], 8, 2, head_dim, 16, "f16", "f16", scale=scale)


@pytest.mark.gpu
def test_rows_of_no_request_are_zeros():
    _, _, _, _, _, out, lse = run_prefill(1, [3, 70], [30, 70], 8, 2, 128, 16, spare_rows=(5, 9))
    for rows in (slice(0, 5), slice(-9, None)):
        assert bool((out[rows] == 0).all()) and bool((lse[rows] == -math.inf).all())
