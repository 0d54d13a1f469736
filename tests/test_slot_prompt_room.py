"""Prompts that a layer has no room for are refused before anything is indexed by them."""
import pytest
import torch

from paper_2604_11001_b200 import slot_time as st


def layer(requests=3, columns=4, positions=50):
    """What prompt_inputs looks at, on the CPU."""
    x = st.Layer.__new__(st.Layer)
    x.torch, x.device, x.columns = torch, torch.device("cpu"), columns
    x.lengths, x.rope = torch.zeros(requests, dtype=torch.int32), torch.zeros(positions, 8)
    x.table = torch.arange(requests * columns, dtype=torch.int32).view(requests, columns)
    x.heads, x.kv_heads, x.head_dim, x.dtype, x.generator = 4, 2, 8, torch.bfloat16, torch.Generator()
    return x


@pytest.mark.parametrize("lengths,chunk", [([51, 1, 1], 0), ([1, 2, 65], 0), ([1, 1, 1, 1], 0), ([1, 1], 0), ([-1, 5, 5], 0), ([], 0), ([5, 5, 5], -1),
                                           ([50, 51, 1], 16), ([0, 0, 0], 0)])
def test_prompts_without_room_are_refused(lengths, chunk):
    with pytest.raises(ValueError, match="prompt"):
        layer().prompt_inputs(lengths, chunk)


def test_pages_bound_them_too():
    with pytest.raises(ValueError, match="prompt"):
        layer(columns=3).prompt_inputs([49, 1, 1])
    assert len(layer(columns=4).prompt_inputs([50, 1, 0], 20)) == 3
