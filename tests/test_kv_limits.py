"""CPU checks of the paged cache's limits: what its kernels could not count is refused before any launch."""
import pytest

from test_kv_host import APPEND, ATTEND, CACHE, EINVAL, EVICT, call

MOST = 2 ** 31 - 2 ** 16
WIDE = dict(table_cols=1 << 27, max_length=MOST)   # (nothing is asked for, so nothing is launched)


def test_lengths_near_2_31_are_refused():
    """Tiles, pages and fours beyond a request's last token are counted in 32 bits."""
    assert call("attend", CACHE, {**ATTEND, **WIDE}) == 0
    assert call("evict", CACHE, {**EVICT, **WIDE, "new_cols": 1 << 27, "max_budget": MOST}) == 0
    for length in (MOST + 1, 2 ** 31 - 64, 2 ** 31 - 1):
        assert call("attend", CACHE, {**ATTEND, **WIDE, "max_length": length}) == EINVAL
        assert call("attend", CACHE, {**ATTEND, **WIDE, "max_length": length, "window": 100}) == EINVAL
        assert call("evict", CACHE, {**EVICT, **WIDE, "max_length": length}) == EINVAL
        assert call("evict", CACHE, {**EVICT, **WIDE, "new_cols": 1 << 27, "max_budget": length}) == EINVAL
        assert call("append", CACHE, {**APPEND, "n_tokens": length, "k": None}) == EINVAL


@pytest.mark.parametrize("heads,head_dim,code", [(1 << 23, 248, 0), (1 << 23, 256, EINVAL), (1 << 30, 64, EINVAL), (2 ** 31 - 8, 8, EINVAL)])
def test_query_rows_of_2_31_elements_are_refused(heads, head_dim, code):
    assert call("attend", {**CACHE, "head_dim": head_dim}, {**ATTEND, "n_heads": heads}) == code
