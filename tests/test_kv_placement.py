"""Which device and stream a call of the key/value cache runs on (no GPU needed: the calls end at
their first look at a tensor, and the devices are stand-ins)."""
import contextlib
import types

import pytest
import torch

CALLS = {"write": lambda kv, c, **more: kv.write(c, Seen, None, None, **more),
         "read": lambda kv, c, **more: kv.read(c, Seen, out=(None, None), **more),
         "attend": lambda kv, c, **more: kv.attend(c, Seen, Seen, **more),
         "select": lambda kv, c, **more: kv.select(c, Seen, Seen, keep=1, **more)}


class Reached(Exception):
    pass


class _Seen:
    """Sequences and queries whose first use ends the call."""

    def __getattr__(self, name):
        raise Reached


Seen = _Seen()


@pytest.fixture
def placed(monkeypatch):
    """(kv, cache on device 1, what has been made current), with device `kv.now` current."""
    from paper_2203_00448_amd import kv
    kv.load_library()
    made = []

    @contextlib.contextmanager
    def device(d):
        made.append(("device", d))
        was, state.now = state.now, d.index
        yield
        state.now = was

    @contextlib.contextmanager
    def stream(s):
        made.append(("stream", s))
        yield

    state = types.SimpleNamespace(now=0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: state.now)
    monkeypatch.setattr(kv, "_device", lambda: state.now)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    cache = types.SimpleNamespace(device=torch.device("cuda", 1), index=1, heads=1, dim=64)
    return kv, cache, made, state


@pytest.mark.parametrize("call", CALLS)
def test_the_cache_s_device_is_current(placed, call):
    kv, cache, made, state = placed
    with pytest.raises(Reached):
        CALLS[call](kv, cache)
    assert ("device", cache.device) in made


@pytest.mark.parametrize("call", CALLS)
def test_nothing_changes_where_it_is_current(placed, call):
    kv, cache, made, state = placed
    state.now = 1
    with pytest.raises(Reached):
        CALLS[call](kv, cache)
    assert not made


@pytest.mark.parametrize("call", CALLS)
def test_a_stream_of_the_cache_s_device(placed, call):
    kv, cache, made, state = placed
    stream = types.SimpleNamespace(device=cache.device)
    with pytest.raises(Reached):
        CALLS[call](kv, cache, stream=stream)
    assert ("device", cache.device) in made and ("stream", stream) in made


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("now", [0, 1])
def test_a_stream_of_another_device_is_refused(placed, call, now):
    kv, cache, made, state = placed
    state.now = now
    with pytest.raises(ValueError):
        CALLS[call](kv, cache, stream=types.SimpleNamespace(device=torch.device("cuda", 0)))


def test_a_status_word_is_reset_on_its_own_device(placed, monkeypatch):
    kv, cache, made, state = placed
    from paper_2203_00448_amd import binding
    word = types.SimpleNamespace(device=cache.device, is_cuda=True, data_ptr=lambda: 4096, numel=lambda: 1)
    reset = []
    stub = types.SimpleNamespace(mp_status_reset=lambda p, s: reset.append((state.now, s.value)) or 0)
    monkeypatch.setattr(binding, "load_library", lambda: stub)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=100 + state.now))
    binding.reset_status(word)
    assert reset == [(1, 101)]
