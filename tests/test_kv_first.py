"""attend over a window and the first tokens, against plain 64-bit forms of its definition."""
import ctypes as C

import pytest
import torch

from kv_common import DT, make_table
from kv_prompt_common import assert_prompt, ref_prompt
from paper_2604_11001_b200 import kvcache as kv
from test_kv_gpu import EDGES, gen, make_cache, randn
from test_kv_host import ATTEND, CACHE, EINVAL, call


def run_first(seed, lengths, heads, n_kv, head_dim, page, dtype, cache, window, first, heads_first=False, weight=False, max_length=None):
    g = gen(seed)
    need = sum(-(-n // page) for n in lengths)
    c = make_cache(g, need + 3, page, n_kv, head_dim, cache, heads_first)
    table, _ = make_table(g, lengths, page, need + 3)
    for r, n in enumerate(lengths):   # what is not seen is not even looked at: wild pages in between
        for i in range(-(-n // page)):
            if window and i * page >= first and (i + 1) * page <= n - window:
                table[r, i] = 2 ** 31 - 1
    q = randn(g, len(lengths), heads, head_dim, dtype=DT[dtype])
    before = c.weight.clone()
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out, lse = c.attend(q, table, ln, window=window, first=first, add_weight=weight, return_lse=True, max_length=max_length)
    c.check()
    starts = list(range(len(lengths) + 1))
    assert_prompt(c, q, starts, table, lengths, out, lse, window=window, first=first)
    if not weight:
        assert torch.equal(before, c.weight)
        return
    _, _, _, reach, rweights = ref_prompt(c, q, starts, table, lengths, window=window, first=first, add=True)
    want, slack = before.double(), before.double().abs() * 2.0 ** -23
    for r, n in enumerate(lengths):
        if n == 0:
            continue
        t = torch.arange(n, device="cuda")
        pg, pl = table[r].long()[t // page], t % page
        ok = pg < c.n_pages
        pg, pl, w = pg[ok], pl[ok], rweights[r].T[ok]
        logit = head_dim * 2.0 ** -23 * reach[r].max() + 2.0 ** -21 * (1 + reach[r].max())
        want[pg, :, pl] += w
        slack[pg, :, pl] += w * (4 * logit + 2.0 ** -20) + 2.0 ** -23 * want[pg, :, pl].abs()
    assert bool(((c.weight.double() - want).abs() <= slack).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("window,first", [(1, 1), (16, 16), (64, 4), (63, 17), (200, 130), (2, 500), (1000, 1)])
def test_first_tokens_stay_visible(dtype, cache, window, first):
    run_first(window, EDGES, 8, 2, 64, 16, dtype, cache, window, first)


@pytest.mark.gpu
@pytest.mark.parametrize("page", [1, 3, 16, 24, 128])
@pytest.mark.parametrize("first", [1, 5, 16, 33])
def test_pages_and_weights(page, first):
    run_first(page + first, [0, 1, 40, 99, 100, 101, 700, 2000], 12, 4, 128, page, "bf16", "bf16", 100, first, heads_first=first % 2 == 0, weight=True)


@pytest.mark.gpu
@pytest.mark.parametrize("lengths", [[20011], [300] * 400, [9000, 1, 0, 17, 8000, 3], [131072]])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_few_and_many_requests(lengths, cache):
    run_first(len(lengths), lengths, 16, 2, 128, 16, "bf16", cache, 256, 7, weight=len(lengths) > 1)


@pytest.mark.gpu
def test_without_a_window_first_has_no_effect_and_with_none_the_bits_are_those_of_the_window():
    g = gen(3)
    c = make_cache(g, 200, 16, 2, 128, "bf16")
    lengths = [3000, 17, 0]
    table, _ = make_table(g, lengths, 16, 200)
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q = randn(g, 3, 8, 128, dtype=torch.bfloat16)
    assert torch.equal(c.attend(q, table, ln), c.attend(q, table, ln, first=9))
    assert torch.equal(c.attend(q, table, ln), c.attend(q, table, ln, window=2999, first=1))
    assert torch.equal(c.attend(q, table, ln, window=100), c.attend(q, table, ln, window=100, first=0))
    assert torch.equal(c.attend(q, table, ln, window=100, first=2 ** 31 - 1), c.attend(q, table, ln))
    assert torch.equal(c.attend(q, table, ln, window=2 ** 31 - 1, first=2 ** 31 - 1), c.attend(q, table, ln))
    c.check()


def test_a_negative_number_of_first_tokens_is_refused():
    assert call("attend", CACHE, {**ATTEND, "first": -1}) == EINVAL
    assert call("attend", CACHE, {**ATTEND, "first": 2 ** 31 - 1, "window": 2 ** 31 - 1}) == 0
    assert kv.fcsim_kv_attend_args.first.offset == C.sizeof(kv.fcsim_kv_attend_args) - 8
