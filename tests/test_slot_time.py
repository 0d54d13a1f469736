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
