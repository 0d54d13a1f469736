"""Prompts in the times of slots, with times that are made up: what they add, exactly."""
import pytest

from paper_2604_11001_b200 import slot_time as st


class Timed:
    """A layer whose times are known: 20 us a slot and 1 ns a token held; 30 us a prompt and 1 us a prompt token, times two in chunks."""
    asked = []

    def __init__(self, lengths, *args, **kw):
        self.lengths, self.cache = lengths, self

    def time(self, repeats=20):
        return 20 + 0.001 * sum(self.lengths)

    def time_prompts(self, lengths, chunk=0, repeats=20):
        Timed.asked.append((lengths, chunk))
        return (30 * len(lengths) + sum(lengths)) * (2 if chunk else 1)

    def check(self):
        pass


@pytest.mark.gpu
@pytest.mark.parametrize("preset", [2, 6])
def test_prompts_are_added_to_every_slot(preset, monkeypatch):
    monkeypatch.setattr(st, "Layer", Timed)
    kw = dict(slots=300, replicas=2, points=3, heads=8, kv_heads=2, head_dim=64)
    plain = st.run(preset, **kw)
    Timed.asked.clear()
    got = st.run(preset, prompts=True, **kw)
    cfg = st.PRESETS[preset](replicas=2, T=300)
    assert plain["rows"] == got["rows"] and (plain["a_us"], plain["b_us"]) == (got["a_us"], got["b_us"])
    assert len(Timed.asked) == 8 * len(cfg.groups)
    for i, (a, b, group) in enumerate(zip(plain["groups"], got["groups"], cfg.groups)):
        asked = Timed.asked[8 * i:8 * i + 8]
        assert a["begun"] == a["prompt_us"] == 0 and b["begun"] > 0
        assert all(chunk == group.chunk and len(lengths) <= max(1, round(b["begun"])) for lengths, chunk in asked)
        tokens, prompts = sum(sum(lengths) for lengths, _ in asked), sum(len(lengths) for lengths, _ in asked)
        assert b["prompt_us"] == pytest.approx((30 + tokens / prompts) * (2 if group.chunk else 1), rel=1e-12)
        more = b["begun"] * b["prompt_us"]
        assert b["slot_us"] == pytest.approx(a["slot_us"] + more, rel=1e-12)
        assert b["tokens_per_second"] == pytest.approx(a["tokens_per_second"] * a["slot_us"] / b["slot_us"], rel=1e-12)
        # every request waits so much longer in each of its slots
        assert b["mean_latency_ms"] - a["mean_latency_ms"] == pytest.approx(more * 1e-3 * b["mean_latency_slots"], rel=1e-6)
