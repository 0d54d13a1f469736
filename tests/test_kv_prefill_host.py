"""CPU checks of prefill's boundary: struct layout, refusals before any launch."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2604_11001_b200 import kvcache as kv
from test_kv_host import CACHE, EINVAL, ESIZE, ROOT
from test_kv_limits import MOST

# Addresses are made up: a call that is refused never reads them, and these calls are all refused or empty.
PREFILL = dict(q=0x1000, out=0x1000, starts=0x1000, table=0x1000, lengths=0x1000, q_row=512, q_head=64, table_row=4, n_rows=0,
               n_requests=0, n_heads=8, dtype=kv.F16, table_cols=4, max_length=64, scale=1.0)


def call(cache, args):
    c, a, need = kv.fcsim_kv_cache(**cache), kv.fcsim_kv_prefill_args(**args), kv.fcsim_kv_workspace()
    lib = kv.load()
    code = lib.fcsim_kv_prefill_workspace(C.byref(c), C.byref(a), C.byref(need))
    if code == 0 and args["n_rows"] > 0:
        return 0      # (what would run is not run here)
    assert lib.fcsim_kv_prefill(C.byref(c), C.byref(a), None, 0, None) == code
    return code


def test_nothing_to_do_is_fine_and_null_is_refused():
    assert call(CACHE, PREFILL) == 0
    assert call(CACHE, {**PREFILL, "q": None, "out": None, "n_requests": 5}) == 0
    lib, c, a, need = kv.load(), kv.fcsim_kv_cache(**CACHE), kv.fcsim_kv_prefill_args(**PREFILL), kv.fcsim_kv_workspace()
    assert lib.fcsim_kv_prefill(None, C.byref(a), None, 0, None) == EINVAL
    assert lib.fcsim_kv_prefill(C.byref(c), None, None, 0, None) == EINVAL
    assert lib.fcsim_kv_prefill_workspace(C.byref(c), C.byref(a), None) == EINVAL
    assert lib.fcsim_kv_prefill_workspace(None, C.byref(a), C.byref(need)) == EINVAL
    assert lib.fcsim_kv_prefill_workspace(C.byref(c), None, C.byref(need)) == EINVAL


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=3), EINVAL), (dict(n_pages=0), EINVAL), (dict(page_size=0), EINVAL), (dict(n_kv_heads=0), EINVAL), (dict(head_dim=63), EINVAL),
    (dict(head_dim=264), EINVAL), (dict(stride_page=-8), EINVAL), (dict(stride_slot=4), EINVAL), (dict(k=None), ESIZE), (dict(k=0x1008), ESIZE),
    (dict(k_scale=0x1000), EINVAL), (dict(dtype=kv.E4M3), EINVAL)])
def test_bad_caches_are_refused(bad, code):
    assert call({**CACHE, **bad}, PREFILL) == code


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=kv.BF16), EINVAL), (dict(dtype=kv.E4M3), EINVAL), (dict(n_rows=-1), EINVAL), (dict(n_rows=MOST + 1), EINVAL), (dict(n_requests=-1), EINVAL),
    (dict(n_requests=65536), EINVAL), (dict(n_requests=65535), 0), (dict(n_heads=0), EINVAL), (dict(n_heads=12), EINVAL), (dict(n_heads=2 ** 31 - 8), EINVAL),
    (dict(max_length=65), EINVAL), (dict(max_length=-1), EINVAL), (dict(table_cols=-1), EINVAL), (dict(table_row=-1), EINVAL), (dict(window=-1), EINVAL),
    (dict(first=-1), EINVAL), (dict(window=2 ** 31 - 1, first=2 ** 31 - 1), 0), (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL),
    (dict(q_row=5), EINVAL), (dict(q_row=-8), EINVAL), (dict(q_head=12), EINVAL), (dict(q_row=0, q_head=0), 0),
    (dict(table_cols=1 << 27, max_length=MOST), 0), (dict(table_cols=1 << 27, max_length=MOST + 1), EINVAL),
    (dict(n_rows=1, q=None), ESIZE), (dict(n_rows=1, out=None), ESIZE), (dict(n_rows=1, q=0x1008), ESIZE), (dict(n_rows=1, out=0x1002), ESIZE),
    (dict(n_rows=1, n_requests=1, starts=None), ESIZE), (dict(n_rows=1, n_requests=1, lengths=None), ESIZE), (dict(n_rows=1, n_requests=1, table=None), ESIZE)])
def test_bad_calls_are_refused(bad, code):
    assert call(CACHE, {**PREFILL, **bad}) == code


@pytest.mark.parametrize("workspace,size", [(None, 0), (None, 1 << 30), (0x1008, 1 << 30), (0x1000, 1000)])
def test_small_or_misplaced_workspaces_are_refused(workspace, size):
    c, a = kv.fcsim_kv_cache(**CACHE), kv.fcsim_kv_prefill_args(**{**PREFILL, "n_rows": 4, "n_requests": 1})
    assert kv.load().fcsim_kv_prefill(C.byref(c), C.byref(a), workspace, size, None) == ESIZE


def test_struct_size(tmp_path):
    src = tmp_path / "s.c"
    src.write_text('#include "fcsim_kv.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu %zu", sizeof(fcsim_kv_prefill_args), '
                   "offsetof(fcsim_kv_prefill_args, table_row), offsetof(fcsim_kv_prefill_args, n_rows), offsetof(fcsim_kv_prefill_args, scale)); return 0; }\n")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "s")], check=True)
    got = subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout.split()
    a = kv.fcsim_kv_prefill_args
    assert [int(x) for x in got] == [C.sizeof(a), a.table_row.offset, a.n_rows.offset, a.scale.offset]
    assert C.sizeof(a) == kv._PREFILL.size
