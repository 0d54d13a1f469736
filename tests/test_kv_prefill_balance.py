"""How prefill's work is divided: few requests of uneven lengths, whose blocks are fewer than CTAs."""
import pytest
import torch

from kv_common import make_table
from kv_prompt_common import assert_prompt
from paper_2604_11001_b200 import kvcache as kv
from test_kv_gpu import gen, make_cache, randn
from test_kv_prefill_values import starts_of, to_int

pytestmark = pytest.mark.gpu

LENGTHS = [1100, 16000, 2100, 900, 7000, 3100, 1500, 4400, 2600, 12000, 1900, 5200, 3700, 800, 6100, 2300]


def median_us(call, n=15):
    flush, times = torch.empty(64 << 20, device="cuda"), []
    for _ in range(n + 3):
        flush.sum()
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b) * 1e3)
    return sorted(times[3:])[n // 2]


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_few_long_blocks_do_not_wait_for_the_longest(cache):
    """16 requests of 7 new tokens each, 8 kv heads: 128 blocks, the longest 3.6 times the mean.  The time is that of the same requests among empty ones, of which
    33 in all are planned for in another way; whole, one a CTA, they took 1.6 (bf16) and 2.3 (e4m3) times as long."""
    g = gen(1)
    c = make_cache(g, sum(-(-n // 64) for n in LENGTHS), 64, 8, 128, cache)
    table, _ = make_table(g, LENGTHS, 64, c.n_pages, fill=0)
    q = randn(g, 16 * 7, 64, 128, dtype=torch.bfloat16)
    few = q, to_int(starts_of([7] * 16)), table, to_int(LENGTHS)
    many = q, to_int(starts_of([7] * 16 + [0] * 17)), torch.cat([table, table.new_zeros(17, table.shape[1])]), to_int(LENGTHS + [0] * 17)
    times = [median_us(lambda: c.prefill(*args)) for args in (few, many)]
    c.check()
    assert times[0] <= 1.3 * times[1], times


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("requests", [4, 9, 16, 17, 33])
@pytest.mark.parametrize("long", [0, 1, 5])
def test_blocks_as_few_as_ctas(cache, requests, long):
    """`long` requests far longer than the others, so that blocks stay whole, are cut into pieces or into equal shares."""
    g = gen(requests)
    lengths = [9000 + 500 * r if r < long else 200 + 97 * r % 1300 for r in range(requests)]
    new = [1 + r % 7 for r in range(requests)]
    c = make_cache(g, sum(-(-n // 16) for n in lengths), 16, 8, 64, cache)
    table, _ = make_table(g, lengths, 16, c.n_pages, fill=0)
    starts = starts_of(new)
    q = randn(g, starts[-1], 32, 64, dtype=torch.bfloat16)
    args = q, to_int(starts), table, to_int(lengths)
    out, lse = c.prefill(*args, return_lse=True)
    c.check()
    assert_prompt(c, q, starts, table, lengths, out, lse)
    assert torch.equal(c.prefill(*args), out)
    assert not bool(next(iter(kv._WORKSPACES[0].values()))[:64 * 1024].any())
