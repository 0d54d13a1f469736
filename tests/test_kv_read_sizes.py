"""read: how 8-bit values are rounded, and rows beyond 2^31 bytes of output."""
import pytest
import torch

from kv_common import DT
from paper_2604_11001_b200 import kvcache as kv
from test_kv_gpu import gen

# Scales whose product with some values lies so near the middle of two values of the output's type that its rounding to 32 bits decides.
SCALES = {"bf16": ["0x1.f95554p+0", "0x1.de6666p+0", "0x1.19b6dcp-1"], "f16": ["0x1.a12aaap+0", "0x1.eb6668p+0", "0x1.8b924ap-1"]}


def products(dtype, device="cpu"):
    """[16, 16, 3] bytes (no NaN), and what read gives for them: the float32 product, rounded."""
    byte = torch.arange(256, dtype=torch.uint8, device=device)
    byte[127] = byte[255] = 0
    raw = byte.view(16, 16, 1).expand(-1, -1, 3).contiguous()
    scale = torch.tensor([float.fromhex(x) for x in SCALES[dtype]], dtype=torch.float32, device=device)
    value = raw.view(torch.float8_e4m3fn).float()
    return raw, scale, (value * scale).to(DT[dtype]), value.double() * scale.double()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_the_scales_tell_both_roundings_apart(dtype):
    _, _, want, exact = products(dtype)
    beside = [(want.view(torch.int16) + i).view(DT[dtype]).double() for i in (-1, 1)]
    nearer = torch.minimum((exact - beside[0]).abs(), (exact - beside[1]).abs()) < (exact - want.double()).abs()
    assert bool(nearer.any(0).any(0).all())      # for every scale some value: rounded once it would be another


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_8_bit_values_are_rounded_to_32_bits_first(dtype):
    raw, scale, want, _ = products(dtype, "cuda")
    rows = raw[..., None].expand(-1, -1, -1, 16).contiguous().view(torch.float8_e4m3fn)      # [pages, places, heads, 16]
    c = kv.PagedKV(rows, rows.clone(), None, scale, scale.flip(0).contiguous())
    k, v = c.read(torch.arange(256, device="cuda"), dtype=DT[dtype])
    c.check()
    value = raw.view(torch.float8_e4m3fn).float()
    assert torch.equal(k, want.view(256, 3, 1).expand(-1, -1, 16))
    assert torch.equal(v, (value * scale.flip(0)).to(DT[dtype]).view(256, 3, 1).expand(-1, -1, 16))


@pytest.mark.gpu
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_rows_behind_2_31_bytes_of_output(cache):
    """All rows of k and v, 5 000 tokens behind the boundary among them."""
    g = gen(3)
    bits = torch.randint(0, 120, (2, 64, 16, 8, 128 * (2 if cache == "bf16" else 1)), generator=g, device="cuda", dtype=torch.uint8)
    pools = bits.view(DT[cache])
    scales = [torch.tensor([0.5 + h for h in range(8)], device="cuda")] * 2 if cache == "e4m3" else [None, None]
    c = kv.PagedKV(pools[0], pools[1], None, *scales)
    edge, more = 1 << 20, 5000
    slots = torch.randint(0, 1024, (edge + more,), generator=g, device="cuda")
    got = c.read(slots)
    c.check()
    assert (got[0].numel() - more * 1024) * 2 == 2 ** 31
    for pool, x in zip(pools, got):
        rows = pool.float().view(1024, 8, 128)
        if cache == "e4m3":
            rows = rows * scales[0][:, None]
        rows = rows.bfloat16().view(torch.int16)
        for at in range(0, edge + more, 1 << 17):
            assert torch.equal(x[at:at + (1 << 17)].view(torch.int16), rows[slots[at:at + (1 << 17)]])
