"""read: what stands at given slots of the cache, bit for bit."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from kv_common import DT
from paper_2604_11001_b200 import kvcache as kv
from test_kv_gpu import gen, make_cache, randn
from test_kv_host import CACHE, EINVAL, ESIZE, ROOT

READ = dict(slots=0x1000, k_out=0x1000, v_out=0x2000, n_tokens=0, dtype=kv.F16)


def plain(pool, scale, slots, page, dtype):
    """Values of slots inside the pool: in 64 bits (exact products), rounded through 32, as the definition has it."""
    x = pool.view(torch.uint8) if pool.dtype == torch.float8_e4m3fn else pool
    x = x[slots // page, slots % page]
    x = x.view(torch.float8_e4m3fn).float() * scale[:, None] if scale is not None else x
    return x.to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("cache", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n_kv,head_dim,page", [(1, 16, 1), (3, 80, 24), (8, 128, 16), (2, 256, 64), (5, 64, 7), (1, 48, 100)])
def test_rows_come_back(cache, dtype, n_kv, head_dim, page):
    g = gen(n_kv)
    for heads_first in (False, True):
        c = make_cache(g, 50, page, n_kv, head_dim, cache, heads_first)
        for n in (1, 2, 37, 50 * page, 3000):
            slots = torch.randint(0, 50 * page, (n,), generator=g, device="cuda")
            k, v = c.read(slots, dtype=DT[dtype])
            assert k.dtype == DT[dtype] and k.shape == (n, n_kv, head_dim)
            assert torch.equal(k, plain(c.k, c.k_scale, slots, page, DT[dtype]))
            assert torch.equal(v, plain(c.v, c.v_scale, slots, page, DT[dtype]))
    c.check()
    k, v = c.read(slots[:0])
    assert k.shape == (0, n_kv, head_dim) and k.dtype == (torch.bfloat16 if cache == "e4m3" else DT[cache])


@pytest.mark.gpu
def test_a_large_read_crosses_2_31_bytes_of_output():
    c = kv.PagedKV.allocate(64, 16, 8, 128)
    c.k.copy_(torch.arange(64 * 16, device="cuda").view(64, 16, 1, 1).expand_as(c.k) % 251)
    n = 1 << 20
    slots = torch.arange(n, device="cuda") % 1024
    k, _ = c.read(slots)
    assert torch.equal(k[:, 0, 0].float(), (slots % 251).float()) and torch.equal(k[-1, -1], k[-1, 0]) and k.numel() * 2 >= 2 ** 31


@pytest.mark.gpu
def test_slots_that_are_none_or_outside():
    c = make_cache(gen(1), 10, 16, 2, 64, "e4m3")
    c.k_scale.fill_(float("nan"))   # (zeros are not scaled)
    slots = torch.tensor([-1, 159, 5, -2 ** 62, 5], device="cuda")
    k, v = c.read(slots)
    c.check()
    assert bool((v[[0, 3]] == 0).all()) and bool((k[[0, 3]] == 0).all()) and bool(torch.isnan(k[[1, 2, 4]].float()).all())
    assert torch.equal(v[[1, 2, 4]], plain(c.v, c.v_scale, slots[[1, 2, 4]], 16, torch.bfloat16))
    k, v = c.read(torch.tensor([160, 0, 2 ** 62, 2 ** 31], device="cuda"))
    assert bool((v[[0, 2, 3]] == 0).all()) and bool((k[[0, 2, 3]] == 0).all())
    with pytest.raises(ValueError, match="page or slot"):
        c.check()


@pytest.mark.gpu
def test_a_request_moves_to_another_cache():
    """Out of pages of 24 in 8 bits, into pages of 16 in 16 bits: attention reads the same values."""
    g = gen(2)
    n, a = 100, make_cache(g, 10, 24, 2, 64, "e4m3")
    b = kv.PagedKV.allocate(10, 16, 2, 64)
    old = torch.arange(5, device="cuda", dtype=torch.int32)[None].contiguous()
    new = torch.arange(7, device="cuda", dtype=torch.int32)[None].contiguous() + 2
    t = torch.arange(n, device="cuda")
    k, v = a.read(old[0, t // 24].long() * 24 + t % 24)
    b.append(None, k, v, None, new[0, t // 16].long() * 16 + t % 16)
    assert torch.equal(b.read(new[0, t // 16].long() * 16 + t % 16)[0], k)
    q = randn(g, 1, 4, 64, dtype=torch.bfloat16)
    ln = torch.tensor([n], dtype=torch.int32, device="cuda")
    x, y = a.attend(q, old, ln).double(), b.attend(q, new, ln).double()
    # k and v were rounded to bf16 (2^-8 relative each): logits (of size 8 here at most) move by 2^-8 of sum |q k|, below 2^-8 * 8 * 8
    assert float((x - y).abs().max()) <= 0.25 * float(x.abs().max())
    a.check(), b.check()


@pytest.mark.gpu
def test_reads_on_streams_and_in_graphs():
    g = gen(4)
    c = make_cache(g, 40, 16, 2, 64, "e4m3")
    slots = torch.randint(0, 640, (300,), generator=g, device="cuda")
    want = c.read(slots)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = c.read(slots)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = c.read(slots)
    slots.copy_(slots.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0].flip(0)) and torch.equal(got[1], want[1].flip(0))


@pytest.mark.gpu
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_outputs_that_begin_at_any_16_bytes(cache):
    c = make_cache(gen(5), 10, 16, 3, 80, cache)
    slots = torch.randint(0, 160, (37,), generator=gen(6), device="cuda")
    want = c.read(slots, dtype=torch.float16)
    for at in (8, 16, 24):
        out = torch.full((2, 37 * 3 * 80 + 64), 7.0, dtype=torch.float16, device="cuda")
        k, v = (x[at:at + 37 * 3 * 80] for x in out)
        args = kv.fcsim_kv_read_args(slots=slots.data_ptr(), k_out=k.data_ptr(), v_out=v.data_ptr(), status=c.status.data_ptr(), n_tokens=37, dtype=kv.F16)
        assert kv.load().fcsim_kv_read(c._c_ref, C.byref(args), torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(k.view_as(want[0]), want[0]) and torch.equal(v.view_as(want[1]), want[1])
        assert bool((out[:, :at] == 7).all()) and bool((out[:, at + 37 * 3 * 80:] == 7).all())
    c.check()


@pytest.mark.gpu
def test_the_binding_refuses():
    c = make_cache(gen(1), 4, 16, 1, 64, "f16")
    slots = torch.zeros(4, dtype=torch.int64, device="cuda")
    for bad, kw in ((slots.int(), {}), (slots.cpu(), {}), (torch.zeros(8, dtype=torch.int64, device="cuda")[::2], {}),
                    (slots, dict(dtype=torch.float32)), (slots, dict(dtype=torch.float8_e4m3fn))):
        with pytest.raises(ValueError):
            c.read(bad, **kw)


@pytest.mark.parametrize("bad,code", [
    (dict(n_tokens=-1), EINVAL), (dict(n_tokens=2 ** 31 - 1), EINVAL), (dict(dtype=kv.E4M3), EINVAL), (dict(dtype=7), EINVAL),
    (dict(n_tokens=1, slots=None), ESIZE), (dict(n_tokens=1, k_out=None), ESIZE), (dict(n_tokens=1, v_out=None), ESIZE),
    (dict(n_tokens=1, k_out=0x1008), ESIZE), (dict(n_tokens=1, v_out=0x1004), ESIZE), (dict(), 0), (dict(dtype=kv.BF16), 0)])
def test_bad_reads_are_refused(bad, code):
    c, a = kv.fcsim_kv_cache(**CACHE), kv.fcsim_kv_read_args(**{**READ, **bad})
    assert kv.load().fcsim_kv_read(C.byref(c), C.byref(a), None) == code
    assert kv.load().fcsim_kv_read(None, C.byref(a), None) == EINVAL
    assert kv.load().fcsim_kv_read(C.byref(c), None, None) == EINVAL


def test_struct_size(tmp_path):
    src = tmp_path / "s.c"
    src.write_text('#include "fcsim_kv.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu", sizeof(fcsim_kv_read_args), '
                   "offsetof(fcsim_kv_read_args, n_tokens)); return 0; }\n")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "s")], check=True)
    got = subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in got] == [C.sizeof(kv.fcsim_kv_read_args), kv.fcsim_kv_read_args.n_tokens.offset]
