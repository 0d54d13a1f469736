"""CPU checks of the paged cache's boundary: exported symbols, struct layout, refusals before any launch."""
import ctypes as C
import os
import re

import pytest

from paper_2604_11001_b200 import kvcache as kv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, ESIZE = -1, -3


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "fcsim_kv.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(fcsim_kv_[a-z_]+)\s*\(", text)))
    assert sorted(kv.EXPORTS) == names
    lib = kv.load()
    for n in names:
        assert hasattr(lib, n), n


def test_struct_sizes(tmp_path):
    """The binding's structs have the header's layout, by the compiler's word."""
    import subprocess
    src = tmp_path / "s.c"
    src.write_text('#include "fcsim_kv.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu %zu %zu %zu %zu\\n", '
                   "sizeof(fcsim_kv_cache), sizeof(fcsim_kv_append_args), sizeof(fcsim_kv_attend_args), "
                   "sizeof(fcsim_kv_evict_args), sizeof(fcsim_kv_workspace), offsetof(fcsim_kv_append_args, eps), "
                   "offsetof(fcsim_kv_attend_args, scale)); return 0; }\n")
    exe = str(tmp_path / "s")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(kv.fcsim_kv_cache), C.sizeof(kv.fcsim_kv_append_args), C.sizeof(kv.fcsim_kv_attend_args),
                   C.sizeof(kv.fcsim_kv_evict_args), C.sizeof(kv.fcsim_kv_workspace), kv.fcsim_kv_append_args.eps.offset,
                   kv.fcsim_kv_attend_args.scale.offset]


# Addresses are made up: a call that is refused never reads them, and these calls are all refused or empty.
CACHE = dict(k=0x1000, v=0x2000, weight=0x3000, k_scale=None, v_scale=None, stride_page=16 * 8 * 64, stride_slot=8 * 64,
             stride_head=64, dtype=kv.F16, n_pages=10, page_size=16, n_kv_heads=8, head_dim=64)
APPEND = dict(q=0x1000, k=0x1000, v=0x1000, q_out=0x1000, q_norm=0x1000, k_norm=0x1000, rope=0x1000, positions=0x1000,
              slots=0x1000, q_row=512, q_head=64, k_row=512, k_head=64, v_row=512, v_head=64, n_tokens=0, n_heads=8,
              dtype=kv.F16, rope_dim=64, n_positions=100, eps=1e-6)
ATTEND = dict(q=0x1000, out=0x1000, table=0x1000, lengths=0x1000, q_row=512, q_head=64, table_row=4, n_requests=0,
              n_heads=8, dtype=kv.F16, table_cols=4, max_length=64, scale=1.0)
EVICT = dict(table=0x1000, lengths=0x1000, budget=0x1000, new_table=0x1000, new_lengths=0x1000, kept=0x1000, table_row=4,
             new_row=2, n_requests=0, table_cols=4, new_cols=2, max_length=64, max_budget=32)


def call(name, cache, args, null_cache=False, null_args=False):
    lib = kv.load()
    c = kv.fcsim_kv_cache(**cache)
    a = {"append": kv.fcsim_kv_append_args, "attend": kv.fcsim_kv_attend_args, "evict": kv.fcsim_kv_evict_args}[name](**args)
    cp, ap = None if null_cache else C.byref(c), None if null_args else C.byref(a)
    if name == "append":
        return lib.fcsim_kv_append(cp, ap, None)
    need = kv.fcsim_kv_workspace()
    code = getattr(lib, f"fcsim_kv_{name}_workspace")(cp, ap, C.byref(need))
    if null_cache or null_args or code != 0:   # the call itself refuses the same things
        assert getattr(lib, f"fcsim_kv_{name}")(cp, ap, None, 0, None) == code
        return code
    return getattr(lib, f"fcsim_kv_{name}")(cp, ap, None, 0, None)


@pytest.mark.parametrize("name,args", [("append", APPEND), ("attend", ATTEND), ("evict", EVICT)])
def test_nothing_to_do_is_fine_and_null_is_refused(name, args):
    assert call(name, CACHE, args) == 0
    assert call(name, CACHE, args, null_cache=True) == EINVAL
    assert call(name, CACHE, args, null_args=True) == EINVAL


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=3), EINVAL), (dict(dtype=-1), EINVAL), (dict(n_pages=0), EINVAL), (dict(page_size=0), EINVAL),
    (dict(n_kv_heads=0), EINVAL), (dict(head_dim=0), EINVAL), (dict(head_dim=63), EINVAL), (dict(head_dim=264), EINVAL),
    (dict(n_pages=1 << 20, page_size=1 << 20), EINVAL), (dict(stride_page=-8), EINVAL), (dict(stride_slot=4), EINVAL),
    (dict(stride_head=65), EINVAL), (dict(k=None), ESIZE), (dict(v=None), ESIZE), (dict(k=0x1008), ESIZE),
    (dict(weight=0x3002), ESIZE), (dict(k_scale=0x1000), EINVAL), (dict(dtype=kv.E4M3), EINVAL),
    (dict(dtype=kv.E4M3, k_scale=0x1000, v_scale=0x1000, head_dim=72, stride_head=80), EINVAL)])
@pytest.mark.parametrize("name,args", [("append", APPEND), ("attend", ATTEND), ("evict", EVICT)])
def test_bad_caches_are_refused(name, args, bad, code):
    assert call(name, {**CACHE, **bad}, args) == code


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=kv.BF16), EINVAL), (dict(dtype=kv.E4M3), EINVAL), (dict(n_tokens=-1), EINVAL), (dict(n_heads=-1), EINVAL),
    (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL), (dict(rope_dim=0), EINVAL),
    (dict(rope_dim=72), EINVAL), (dict(rope_dim=24), EINVAL), (dict(rope_dim=7, interleaved=1), EINVAL),
    (dict(n_positions=0), EINVAL), (dict(q_row=5), EINVAL), (dict(k_head=-64), EINVAL), (dict(v_row=12), EINVAL),
    (dict(n_tokens=1, k=None), ESIZE), (dict(n_tokens=1, v=None), ESIZE), (dict(n_tokens=1, slots=None), ESIZE),
    (dict(n_tokens=1, positions=None), ESIZE), (dict(n_tokens=1, q=None), ESIZE), (dict(n_tokens=1, q_out=None), ESIZE),
    (dict(n_tokens=1, q=0x1004), ESIZE), (dict(n_tokens=1, q_norm=0x1002), ESIZE), (dict(rope=0x1001), ESIZE)])
def test_bad_appends_are_refused(bad, code):
    assert call("append", CACHE, {**APPEND, **bad}) == code


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=kv.BF16), EINVAL), (dict(n_requests=-1), EINVAL), (dict(n_heads=0), EINVAL), (dict(n_heads=12), EINVAL),
    (dict(table_cols=-1), EINVAL), (dict(max_length=-1), EINVAL), (dict(max_length=65), EINVAL), (dict(window=-1), EINVAL),
    (dict(table_row=-4), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL),
    (dict(q_row=3), EINVAL), (dict(q_head=-64), EINVAL), (dict(n_requests=1, q=None), ESIZE),
    (dict(n_requests=1, out=None), ESIZE), (dict(n_requests=1, lengths=None), ESIZE), (dict(n_requests=1, table=None), ESIZE),
    (dict(n_requests=1, q=0x1002), ESIZE), (dict(n_requests=1, out=0x1008), ESIZE)])
def test_bad_attends_are_refused(bad, code):
    assert call("attend", CACHE, {**ATTEND, **bad}) == code


def test_attend_weights_need_a_place():
    assert call("attend", {**CACHE, "weight": None}, {**ATTEND, "n_requests": 1, "add_weight": 1}) == ESIZE
    # a workspace that is missing or too small
    c, a = kv.fcsim_kv_cache(**CACHE), kv.fcsim_kv_attend_args(**{**ATTEND, "n_requests": 1, "add_weight": 1})
    assert kv.load().fcsim_kv_attend(C.byref(c), C.byref(a), None, 0, None) == ESIZE
    assert kv.load().fcsim_kv_attend(C.byref(c), C.byref(a), 0x1000, 16, None) == ESIZE
    assert kv.load().fcsim_kv_attend_workspace(C.byref(c), C.byref(a), None) == EINVAL


@pytest.mark.parametrize("bad,code", [
    (dict(n_requests=-1), EINVAL), (dict(max_length=65), EINVAL), (dict(max_length=-1), EINVAL), (dict(max_budget=33), EINVAL),
    (dict(max_budget=-1), EINVAL), (dict(recent=-1), EINVAL), (dict(first=-1), EINVAL), (dict(table_row=-1), EINVAL),
    (dict(new_row=-1), EINVAL), (dict(n_requests=1, lengths=None), ESIZE), (dict(n_requests=1, budget=None), ESIZE),
    (dict(n_requests=1, new_lengths=None), ESIZE), (dict(n_requests=1, table=None), ESIZE),
    (dict(n_requests=1, new_table=None), ESIZE), (dict(n_requests=1, kept=None), ESIZE)])
def test_bad_evictions_are_refused(bad, code):
    assert call("evict", CACHE, {**EVICT, **bad}) == code


def test_eviction_needs_weights():
    assert call("evict", {**CACHE, "weight": None}, EVICT) == ESIZE


def test_the_binding_refuses_cpu_tensors():
    import torch
    k = torch.zeros(2, 16, 1, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        kv.PagedKV(k, k)


def test_active_sets_hold_the_usage_they_are_drawn_for():
    import numpy as np

    from paper_2604_11001_b200 import slot_time as st
    from paper_2604_11001_b200 import workloads as wl
    for cfg, usage in ((wl.config1(), 3000), (wl.config6(), 16492), (wl.config2(), 65536)):
        lengths = st.active_set(cfg, usage, np.random.default_rng(1))
        assert min(lengths) >= 1 and len(lengths) <= cfg.Acap
        assert sum(lengths) == usage or len(lengths) == cfg.Acap
        most = max(t.vmax for t in cfg.prompt) + max(t.vmax for t in cfg.decode)
        assert max(lengths) < most
        assert max(st.active_set(cfg, usage, np.random.default_rng(1), limit=40)) <= 40
