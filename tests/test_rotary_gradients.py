"""Rotary positions and tensors that want a gradient (no GPU needed: the calls end before they look at a
device): the turn builds no graph, so a call that would lose one is refused."""
import types

import pytest
import torch

from test_kv_placement import placed  # noqa: F401


def call(placed, **which):  # noqa: F811
    from paper_2203_00448_amd import rotary
    rotary.load_library()
    _, handle, _, state = placed
    state.now = 1
    rows = {name: torch.zeros(3, 2, 8, requires_grad=name in which) for name in ("q", "k", "out", "k_out")}
    handle = types.SimpleNamespace(device=handle.device, index=1, turned=8, pairs=False, magnitude=1.0, _freq=0)
    rotary.rotate(handle, torch.zeros(3, dtype=torch.int32), rows.pop("q"), rows.pop("k"), **rows)


@pytest.mark.parametrize("which", ["q", "k", "out", "k_out"])
def test_a_graph_is_not_lost(placed, which):  # noqa: F811
    with pytest.raises(ValueError, match="inverse"):
        call(placed, **{which: True})


@pytest.mark.parametrize("which", ["q", "k", "out", "k_out"])
def test_without_a_graph_to_lose(placed, which):  # noqa: F811
    with torch.no_grad(), pytest.raises(ValueError, match="position"):
        call(placed, **{which: True})
    with pytest.raises(ValueError, match="position"):
        call(placed)
