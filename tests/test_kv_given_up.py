"""A wait that was given up leaves the workspaces wrong, which all caches of a device share: each cache's check() tells of it.  (The bit is set from here: no
wait runs out.)"""
import gc

import pytest
import torch

from paper_2604_11001_b200 import kvcache as kv
from test_kv_prefill_values import setting

pytestmark = pytest.mark.gpu


def told(cache):
    with pytest.raises(RuntimeError, match="given up"):
        cache.check()


def test_every_cache_tells_of_it_once():
    (a, *args), (b, *_), (c, *_) = (setting(i, [700, 40], [30, 40]) for i in range(3))
    for cache in (a, b, c):
        cache.check()
    want = a.prefill(*args)
    c.status.fill_(kv.BAD_PAGE)
    a.status.fill_(kv.STUCK)
    told(b)                              # first one that has not met it
    assert not b._workspaces
    d, *_ = setting(4, [9], [9])         # made afterwards: nothing to tell
    d.check()
    assert torch.equal(a.prefill(*args), want)
    told(a)
    told(c)                              # (what else its word held was of calls before)
    for cache in (a, b, c, d):
        cache.check()


def test_a_cache_that_is_gone():
    (a, *_), (b, *_) = setting(1, [40], [40]), setting(2, [40], [40])
    a.status.fill_(kv.STUCK)
    del a
    gc.collect()
    told(b)
    b.check()


def test_other_bits_stay_with_their_cache():
    (a, *_), (b, *_) = setting(1, [40], [40]), setting(2, [40], [40])
    a.status.fill_(kv.BAD_LENGTH)
    b.check()
    with pytest.raises(ValueError, match="length"):
        a.check()
    gone = len(kv._STATUS[0])
    for i in range(20):
        setting(i, [5], [5])[0].status.fill_(kv.BAD_PAGE)
    gc.collect()
    a.check()
    assert len(kv._STATUS[0]) <= gone    # words of caches that are gone are dropped
