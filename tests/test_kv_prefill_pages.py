"""prefill over tables in which whole tiles of keys have no page in the pool, against plain 64-bit forms: which keys a tile holds is told to the
softmax apart from the copies, and nothing is copied for such a tile."""
import pytest
import torch

from kv_common import DT, make_table
from kv_prompt_common import assert_prompt
from test_kv_gpu import gen, make_cache, randn
from test_kv_prefill_values import starts_of, to_int

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("head_dim", [64, 128, 256])
@pytest.mark.parametrize("page", [8, 12, 64, 128])
def test_tiles_of_keys_without_a_page(dtype, cache, head_dim, page):
    """Every other tile or so of 128 tokens wholly outside the pool, some single pages besides: from tile to tile, and from what stood at its place
    eight tiles before, the keys that count are others.  More blocks than CTAs, in runs that go on over their borders."""
    g = gen(page + head_dim)
    new = [1 + 37 * r % 150 for r in range(40)]
    lengths = [new[r] + 1000 + 211 * r % 1500 for r in range(40)]
    n_pages = sum(-(-n // page) for n in lengths) + 1
    c = make_cache(g, n_pages, page, 2, head_dim, cache)
    table, _ = make_table(g, lengths, page, n_pages)
    rows, cols = table.shape
    tile = torch.arange(cols, device="cuda") * page // 128
    tiles = torch.rand(rows, int(tile[-1]) + 1, generator=g, device="cuda") < 0.4
    table[tiles[:, tile] | (torch.rand(rows, cols, generator=g, device="cuda") < 0.05)] = n_pages
    starts = starts_of(new)
    q = randn(g, starts[-1], 4, head_dim, dtype=DT[dtype])
    args = to_int(starts), table, to_int(lengths)
    out, lse = c.prefill(q, *args, return_lse=True)
    assert_prompt(c, q, starts, table, lengths, out, lse)
    for _ in range(5):
        assert torch.equal(c.prefill(q, *args), out)
    with pytest.raises(ValueError, match="page"):
        c.check()
