"""The sum of a row's weights over long contexts, where one CTA walks over all of them."""
import math

import pytest
import torch

from kv_common import DT
from paper_2604_11001_b200 import kvcache as kv
from test_kv_prefill_values import starts_of, to_int
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
