"""Prompts and windows in the times of slots: what a layer attends over, what it counts."""
import sys

import pytest
import torch

from kv_prompt_common import assert_prompt
from paper_2604_11001_b200 import slot_time as st

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("chunk,window", [(0, 0), (64, 0), (7, 0), (0, 30), (50, 30)])
def test_prompts_of_a_layer_are_attended_over(cache, chunk, window):
    lengths = [130, 1, 64, 77]
    layer = st.Layer(lengths, heads=8, kv_heads=2, head_dim=64, cache=cache, spare=1, window=window)
    inputs = layer.prompt_inputs(lengths, chunk)
    assert len(inputs) == (1 if chunk == 0 else -(-130 // chunk))
    for i, part in enumerate(inputs):
        out, = layer.prompts([part])
        q, k, v, positions, slots, starts, upto = part
        # (the rotation that append gives q is append's own: the same call again, its tokens to the same places)
        q = layer.cache.append(q, k, v, positions, slots, rope=layer.rope, q_norm=layer.norm, k_norm=layer.norm)
        again, lse = layer.cache.prefill(q, starts, layer.table, upto, window=window, first=st.FIRST, return_lse=True)
        assert torch.equal(out, again)
        assert_prompt(layer.cache, q, starts.tolist(), layer.table, upto.tolist(), out, lse, window=window, first=st.FIRST)
        assert upto.tolist() == [min(n, (i + 1) * chunk if chunk else n) for n in lengths]
    layer.cache.check()
    assert layer.time_prompts(lengths, chunk, repeats=2) > 0
    assert layer.lengths.tolist() == lengths
    layer.grow()                                       # and the slots go on behind them
    layer.cache.check()


def test_a_window_shortens_what_is_read():
    """131 072 tokens, of which a window of 256 leaves 260: less than half of the time."""
    lengths = [4096] * 32
    times = [st.Layer(lengths, heads=16, kv_heads=4, head_dim=128, spare=1, window=w).time(10) for w in (0, 256)]
    assert times[1] < 0.5 * times[0]


@pytest.mark.parametrize("preset,budget,window", [(2, None, 0), (6, 32, 64)])
def test_slots_with_prompts_take_longer(preset, budget, window):
    """The same run and the same sets: to every slot the admitted requests' prompts are added."""
    kw = dict(slots=300, replicas=2, points=2, budget=budget, window=window, heads=8, kv_heads=2, head_dim=64)
    got = st.run(preset, prompts=True, **kw)
    for g in got["groups"]:
        assert g["begun"] > 0 and g["prompt_us"] > 0
        # the slot's own part is a + b U, above zero
        assert g["slot_us"] > g["begun"] * g["prompt_us"]
    plain = st.run(preset, **kw)
    assert all(g["begun"] == 0 and g["prompt_us"] == 0 for g in plain["groups"])


def test_the_command_counts_prompts(monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["slot_time", "--preset", "6", "--slots", "100", "--replicas", "2", "--heads", "4", "--kv-heads", "2", "--head-dim", "64",
                                      "--prompts", "--window", "128"])
    st.main()
    assert "requests begin in a slot" in capsys.readouterr().out
