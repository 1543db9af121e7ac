"""Host-side checks of the 4-bit cache, the blocks for requests and the rotary positions (no GPU needed):
bad arguments are refused before anything is launched."""
import ctypes

import pytest

from test_kv_abi import Call

AT = 1 << 20  # an address that is never dereferenced


@pytest.fixture(scope="module")
def kv():
    from paper_2203_00448_amd import kv
    kv.load_library()
    return kv


def call4(kv):
    c = Call(kv)
    c.cache = kv._CacheArg(AT, AT, AT, AT, None, None, 100, 4, 128, 64, kv.E2M1)
    return c


@pytest.mark.parametrize("change", [
    {"cache__kind": 3}, {"cache__kind": 5}, {"cache__dim": 96}, {"cache__dim": 32}, {"cache__block": 8},
    {"cache__k_code": None}, {"cache__v_code": None}, {"cache__k_exp": None}, {"cache__v_exp": None},
    {"cache__k_code": AT + 8}, {"cache__v_code": AT + 8}, {"cache__k_exp": AT + 8}, {"cache__v_exp": AT + 4},
    {"cache__mean_code": AT}, {"cache__mean_exp": AT}, {"seqs__longest": 641}, {"seqs__n_tokens": 1 << 31},
    {"status": None}])
def test_cache_refusals(kv, change):
    c = call4(kv)
    for path, value in change.items():
        *where, name = path.split("__")
        setattr(getattr(c, where[0]) if where else c, name, value)
    for call in ("write", "read", "attend"):
        assert getattr(c, call)() == -1, (call, change)


def test_no_selection_of_4_bits(kv):
    c = call4(kv)
    assert c.select() == -1
    c.blocks, c.keep = ctypes.c_void_p(AT), 4
    assert c.attend() == -1
    assert c.size(kv.OP_SELECT) == 0 and c.size(kv.OP_ATTEND) == 0
    c.keep = 0
    c.seqs.table_stride = c.seqs.table_width = 1 << 16
    c.seqs.longest = 1 << 22
    need = c.size(kv.OP_ATTEND)
    assert need > 0
    c.blocks, c.room = None, need - 1
    assert c.attend() == -1


def test_rows_of_calls_that_no_launch_holds(kv):
    c = call4(kv)
    c.cache.heads, c.q_heads = 1 << 16, 1 << 16
    c.seqs.n_tokens = c.seqs.most_new = 1 << 30
    assert c.attend() == -1


@pytest.fixture(scope="module")
def pages():
    from paper_2203_00448_amd import pages
    pages.load_library()
    return pages


EXTEND = dict(ids=AT, n_ids=100, used=AT, table=AT, stride=10, width=10, block=64, length=AT, more=AT, n_seqs=3,
              n_tokens=30, length_out=AT, used_out=AT, begin=AT, position=AT, slot=AT, ws=AT, room=1 << 20, status=AT)
RELEASE = dict(ids=AT, n_ids=100, used=AT, table=AT, stride=10, width=10, block=64, length=AT, done=AT, n_seqs=3,
               length_out=AT, used_out=AT, ws=AT, room=1 << 20, status=AT)
SHARED = [{"ids": None}, {"n_ids": -1}, {"n_ids": 1 << 31}, {"used": None}, {"table": None}, {"stride": 9},
          {"stride": 1 << 62}, {"width": -1}, {"width": 1 << 31}, {"block": 0}, {"block": 48}, {"block": 128},
          {"length": None}, {"n_seqs": -1}, {"n_seqs": 1 << 31}, {"length_out": None}, {"used_out": None}, {"ws": None},
          {"ws": AT + 8}, {"room": 39}, {"room": 0}, {"status": None}]


@pytest.mark.parametrize("change", SHARED + [{"more": None}, {"begin": None}, {"n_tokens": -1}, {"n_tokens": 1 << 31}])
def test_extend_refusals(pages, change):
    assert pages.load_library().mp_kv_extend(*(EXTEND | change).values(), None) == -1


@pytest.mark.parametrize("change", SHARED + [{"done": None}, {"n_seqs": 1 << 29}])
def test_release_refusals(pages, change):
    # 2^29 sequences: a launch has fewer than 2^32 threads
    assert pages.load_library().mp_kv_release(*(RELEASE | {"room": 1 << 40} | change).values(), None) == -1


def test_pages_workspace(pages):
    size = pages.load_library().mp_kv_pages_workspace_size
    assert size(0) == 16 and size(3) == 40 and size(-1) == 0 and size((1 << 30) + 1) == 0


@pytest.fixture(scope="module")
def rotary():
    from paper_2203_00448_amd import rotary
    rotary.load_library()
    return rotary


@pytest.mark.parametrize("change", [
    {"position": None}, {"position": AT + 2}, {"n_tokens": -1}, {"n_tokens": 1 << 31}, {"freq": None}, {"freq": AT + 4},
    {"turned": 0}, {"turned": -2}, {"turned": 3}, {"turned": 130}, {"layout": 2}, {"layout": -1}, {"dim": 1},
    {"dim": 8192}, {"q": None}, {"q_out": None}, {"k": None}, {"k_out": None}, {"q_heads": 0}, {"q_heads": 1 << 17},
    {"k_heads": -1}, {"k_heads": 1 << 17}, {"q__data": None}, {"q__dtype": 3}, {"q__dtype": 1}, {"k__dtype": 2},
    {"q_out__dtype": 1}, {"k_out__dtype": 1}, {"q__token_stride": -1}, {"k__head_stride": 1 << 60}, {"q__data": AT + 1},
    {"q_out__token_stride": 0}, {"q_out__head_stride": 127}, {"k_out__head_stride": 0}])
def test_rotate_refusals(kv, rotary, change):
    rows = {name: kv._RowsArg(AT, 8 * 128, 128, 0) for name in ("q", "q_out", "k", "k_out")}
    args = dict(position=AT, n_tokens=5, freq=AT, turned=128, layout=0, magnitude=1.0, inverse=0, dim=128, q="q",
                q_heads=8, q_out="q_out", k="k", k_heads=2, k_out="k_out")
    for path, value in change.items():
        if "__" in path:
            where, name = path.split("__")
            setattr(rows[where], name, value)
        else:
            args[path] = value
    args = [ctypes.addressof(rows[x]) if isinstance(x, str) else x for x in args.values()]
    assert rotary.load_library().mp_rotate(*args, None) == -1


def test_python_refuses_host_tensors(kv, pages, rotary):
    import torch
    with pytest.raises(TypeError):
        kv.new_cache(4, 2, 64, kind=kv.E2M1, device="cpu")
    with pytest.raises(TypeError):
        pages.new_pool(4, device="cpu")
    with pytest.raises(TypeError):
        rotary.Rotation(64, device="cpu")
    with pytest.raises(ValueError):
        rotary.Rotation(63, device="cpu")
    assert torch.zeros(1).device.type == "cpu"
