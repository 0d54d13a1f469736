"""Slots of simulated systems on a real cache: what a layer has room for, what is timed, what the figures mean."""
import pytest

from paper_2604_11001_b200 import slot_time as st


@pytest.mark.gpu
@pytest.mark.parametrize("budget", [None, 40])
def test_a_layer_grows_by_its_spare_slots_and_no_further(budget):
    """Past them the table, or the positions, would end: refused on the host."""
    layer = st.Layer([5, 33, 16], heads=4, kv_heads=2, head_dim=64, cache="f16", budget=budget, spare=70)
    for _ in range(70):
        layer.grow()
    assert layer.positions.tolist() == [75, 103, 86]
    assert layer.time(1) > 0                           # one more slot can still be timed
    with pytest.raises(ValueError, match="spare"):
        layer.grow()
    assert layer.positions.tolist() == [75, 103, 86]


@pytest.mark.gpu
@pytest.mark.parametrize("budget", [None, 32])
def test_sets_grow_by_as_many_slots_as_are_asked_for(budget):
    got = st.run(6, slots=200, replicas=4, points=2, grow=400, budget=budget, heads=4, kv_heads=2, head_dim=64, cache="f16")
    assert len(got["rows"]) >= 1


@pytest.mark.gpu
@pytest.mark.parametrize("budget", [None, 48])
def test_timing_a_slot_leaves_the_layer_as_it_was(budget):
    import torch
    layer = st.Layer([5, 33, 16, 48], heads=4, kv_heads=2, head_dim=64, cache="f16", budget=budget, spare=4)
    layer.grow()
    t = torch.cat([torch.arange(n) for n in layer.lengths.tolist()]).cuda()
    r = torch.repeat_interleave(torch.arange(4, device="cuda"), layer.lengths.long())
    held = lambda: [x.view(-1, 2, 64)[layer._slots(r, t)].clone() for x in (layer.cache.k, layer.cache.v)] \
        + [layer.lengths.clone(), layer.positions.clone()] + ([layer.cache.weight.clone()] if budget else [])  # noqa: E731
    before = held()
    assert layer.time(3) > 0
    assert all(torch.equal(a, b) for a, b in zip(before, held()))
    layer.grow()                                       # the pages have room for the next slot all the same
    layer.cache.check()


def test_a_budget_cuts_the_requests_that_there_are():
    """It takes no others in: the number of requests and their order are those of the uncut set."""
    import numpy as np

    from paper_2604_11001_b200 import workloads as wl
    for cfg, usage in ((wl.config2(), 8000), (wl.config2(), 65536), (wl.config5(), 100000), (wl.config6(), 16492)):
        whole = st.active_set(cfg, usage, np.random.default_rng(1))
        cut = st.active_set(cfg, usage, np.random.default_rng(1), limit=40)
        assert cut == [min(n, 40) for n in whole]
        assert sum(whole) == usage or len(whole) == cfg.Acap


@pytest.mark.gpu
def test_a_smaller_budget_takes_less_time():
    """Predicted from the same simulated run: its usages, its requests, less of each on the GPU; the cuts are in the time."""
    got = [st.run(2, slots=600, replicas=2, points=4, budget=b) for b in (None, 512, 64)]
    for g, budget in zip(got[1:], (512, 64)):
        assert [(r["usage"], r["requests"]) for r in g["rows"]] == [(r["usage"], r["requests"]) for r in got[0]["rows"]]
        assert all(r["held"] < r["requests"] * (budget + st.SLACK) for r in g["rows"])
        assert any(r["cuts_us"] > 0 for r in g["rows"]) and all(r["us"] > r["cuts_us"] for r in g["rows"])
        assert [x["mean_latency_slots"] for x in g["groups"]] == [x["mean_latency_slots"] for x in got[0]["groups"]]
    times = [[x["slot_us"] for x in g["groups"]] for g in got]
    for i in range(2):
        assert times[2][i] < times[0][i]
    assert got[2]["rows"][-1]["us"] < got[0]["rows"][-1]["us"]


@pytest.mark.gpu
def test_timing_cuts_leaves_the_layer_as_it_was():
    import torch
    layer = st.Layer([5, 40, 70] + [60] * 130, heads=4, kv_heads=2, head_dim=64, cache="f16", budget=40, spare=2)
    t = torch.cat([torch.arange(n) for n in layer.lengths.tolist()]).cuda()
    r = torch.repeat_interleave(torch.arange(layer.lengths.numel(), device="cuda"), layer.lengths.long())
    held = lambda: [x.view(-1, 2, 64)[layer._slots(r, t)].clone() for x in (layer.cache.k, layer.cache.v)] \
        + [layer.cache.weight.transpose(1, 2).reshape(-1, 2)[layer._slots(r, t)].clone(), layer.lengths.clone(), layer.table.clone()]  # noqa: E731
    before = held()
    assert layer.time_cuts(3) > 0
    assert all(torch.equal(a, b) for a, b in zip(before, held()))
    layer.grow()
    layer.cache.check()
    assert st.Layer([5, 6], heads=4, kv_heads=2, head_dim=64, cache="f16", budget=40).time_cuts() == 0.0


def test_latencies_are_the_times_of_a_requests_own_slots():
    """Idle slots before and after a request are none of its latency, full ones in it are."""
    import numpy as np
    seconds = np.array([1.0, 1.0, 7.0, 7.0, 1.0, 1.0, 2.0, 1.0])
    done, latency = np.array([4, 7, 3, 8]), np.array([2, 1, 1, 8])
    assert st.latency_seconds(seconds, done, latency).tolist() == [14.0, 2.0, 7.0, 21.0]
    assert st.latency_seconds(seconds, done[:0], latency[:0]).size == 0


@pytest.mark.gpu
def test_results_in_seconds_follow_from_the_runs_own_slots():
    """A system that is idle half of the time, replayed request by request from its trace and log."""
    import numpy as np

    from paper_2604_11001_b200 import binding as fb
    from paper_2604_11001_b200 import workloads as wl
    preset = lambda replicas, T: wl.config6(replicas=replicas, T=T, total_rate=0.02)  # noqa: E731
    old = st.PRESETS.get(6)
    st.PRESETS[6] = preset
    try:
        got = st.run(6, slots=3000, replicas=4, points=3, heads=4, kv_heads=2, head_dim=64, cache="f16")
    finally:
        st.PRESETS[6] = old
    cfg = preset(4, 3000).with_(complog_cap=3000)
    sim = fb.Simulation(cfg)
    sim.run(3000)
    counters, _ = sim.stats()
    usage, log = sim.trace()[:, :, 0].cpu().numpy(), sim.complog().cpu().numpy()
    sim.close()
    assert 0.1 < (usage == 0).mean() < 0.9
    for g, mine in enumerate(np.split(np.arange(cfg.n_replicas), len(cfg.groups))):
        waits, total = [], 0.0
        for r in mine:
            us = got["a_us"] + got["b_us"] * usage[r]
            total += us.sum()
            for done, latency in log[r, :counters[r, fb.COUNTER_NAMES.index("n_logged")]]:
                waits.append(sum(us[done - latency:done]))
        one = got["groups"][g]
        assert one["mean_latency_ms"] == pytest.approx(np.mean(waits) * 1e-3, rel=1e-9)
        assert one["slot_us"] == pytest.approx(total / (len(mine) * 3000), rel=1e-9)
        tokens = counters[mine, fb.COUNTER_NAMES.index("tokens_generated")].sum()
        assert one["tokens_per_second"] == pytest.approx(tokens / (total * 1e-6), rel=0.1)
