"""Which device and stream the calls for pages and rotary positions run on (no GPU needed: the calls end
at their first look at a tensor, and the devices are stand-ins)."""
import types

import pytest
import torch

from test_kv_placement import Reached, Seen, placed  # noqa: F401


def calls(handle):
    from paper_2203_00448_amd import pages, rotary
    pages.load_library(), rotary.load_library()
    return {"extend": lambda **more: pages.extend(handle, Seen, Seen, Seen, step=Seen, **more),
            "release": lambda **more: pages.release(handle, Seen, Seen, Seen, **more),
            "rotate": lambda **more: rotary.rotate(handle, Seen, Seen, **more)}


@pytest.mark.parametrize("call", ["extend", "release", "rotate"])
def test_the_handle_s_device_is_current(placed, call):  # noqa: F811
    kv, handle, made, state = placed
    with pytest.raises(Reached):
        calls(handle)[call]()
    assert ("device", handle.device) in made
    made.clear()
    state.now = 1
    with pytest.raises(Reached):
        calls(handle)[call]()
    assert not made
    stream = types.SimpleNamespace(device=handle.device)
    with pytest.raises(Reached):
        calls(handle)[call](stream=stream)
    assert ("device", handle.device) in made and ("stream", stream) in made


@pytest.mark.parametrize("call", ["extend", "release", "rotate"])
@pytest.mark.parametrize("now", [0, 1])
def test_a_stream_of_another_device_is_refused(placed, call, now):  # noqa: F811
    kv, handle, made, state = placed
    state.now = now
    with pytest.raises(ValueError):
        calls(handle)[call](stream=types.SimpleNamespace(device=torch.device("cuda", 0)))
