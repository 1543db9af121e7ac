"""Host-side checks of the key/value cache's entry points (no GPU needed): bad
arguments are refused before anything is launched."""
import ctypes

import pytest

from kv_defs import E4M3_VALUES, encode, least_exponent


@pytest.fixture(scope="module")
def kv():
    from paper_2203_00448_amd import kv
    kv.load_library()
    return kv


class Call:
    """Arguments that would pass, on addresses that are never dereferenced; one or more are
    changed before a call that has to fail a check."""

    def __init__(self, kv):
        self.kv, self.lib = kv, kv.load_library()
        at = 1 << 20
        self.cache = kv._CacheArg(at, at, at, at, at, at, 100, 4, 128, 64, 0)
        self.seqs = kv._SeqsArg(at, 10, 10, at, at, 3, 30, 30, 640)
        self.k = kv._RowsArg(at, 512, 128, 0)
        self.v = kv._RowsArg(at, 512, 128, 0)
        self.q = kv._RowsArg(at, 1024, 128, 0)
        self.o = kv._RowsArg(at, 1024, 128, 0)
        self.p = ctypes.c_void_p(at)
        self.q_heads, self.blocks, self.keep, self.first, self.recent = 8, None, 0, 1, 1
        self.out, self.ws, self.room, self.status = self.p, self.p, 1 << 40, self.p

    def _a(self, x):
        return None if x is None else ctypes.addressof(x)

    def write(self):
        return self.lib.mp_kv_write(self._a(self.cache), self._a(self.seqs), self._a(self.k), self._a(self.v),
                                    self.status, None)

    def read(self):
        return self.lib.mp_kv_read(self._a(self.cache), self._a(self.seqs), self._a(self.k), self._a(self.v),
                                   self.status, None)

    def attend(self):
        return self.lib.mp_kv_attend(self._a(self.cache), self._a(self.seqs), self._a(self.q), self.q_heads, 0.1,
                                     self.blocks, self.keep, self._a(self.o), None, self.ws, self.room, self.status,
                                     None)

    def select(self):
        return self.lib.mp_kv_select(self._a(self.cache), self._a(self.seqs), self._a(self.q), self.q_heads,
                                     self.keep or 4, self.first, self.recent, self.out, self.ws, self.room,
                                     self.status, None)

    def size(self, op):
        return self.lib.mp_kv_workspace_size(op, self._a(self.cache), self._a(self.seqs), self.q_heads, self.keep)


CALLS = ("write", "read", "attend", "select")


def refused(kv, calls, **changes):
    c = Call(kv)
    for path, value in changes.items():
        *where, name = path.split("__")
        setattr(getattr(c, where[0]) if where else c, name, value)
    for call in calls:
        assert getattr(c, call)() == -1, (call, changes)


@pytest.mark.parametrize("change", [
    {"cache": None}, {"seqs": None}, {"status": None},
    {"cache__n_blocks": 0}, {"cache__n_blocks": 1 << 31}, {"cache__heads": 0}, {"cache__heads": 1 << 17},
    {"cache__dim": 96}, {"cache__dim": 0}, {"cache__block": 8}, {"cache__block": 128}, {"cache__kind": 2},
    {"cache__k_code": None}, {"cache__v_code": None}, {"cache__k_exp": None}, {"cache__v_exp": None},
    {"cache__mean_code": None}, {"cache__mean_exp": None},
    {"cache__k_code": (1 << 20) + 8}, {"cache__v_code": (1 << 20) + 4}, {"cache__mean_code": (1 << 20) + 1},
    {"seqs__n_seqs": -1}, {"seqs__n_seqs": 1 << 31}, {"seqs__n_tokens": -1}, {"seqs__n_tokens": 1 << 31},
    {"seqs__table_width": -1}, {"seqs__table_stride": 9}, {"seqs__table_stride": 1 << 62},
    {"seqs__most_new": -1}, {"seqs__longest": -1}, {"seqs__longest": 641}, {"seqs__table": None},
    {"seqs__length": None}, {"seqs__begin": None}])
def test_shared_refusals(kv, change):
    refused(kv, CALLS, **change)


@pytest.mark.parametrize("change", [
    {"k": None}, {"v": None}, {"k__data": None}, {"v__data": None}, {"k__dtype": 3}, {"v__dtype": -1},
    {"k__token_stride": -1}, {"k__head_stride": -1}, {"v__token_stride": 1 << 60}, {"v__head_stride": 1 << 60},
    {"k__data": (1 << 20) + 1}])
def test_rows_refusals(kv, change):
    refused(kv, ("write", "read"), **change)


@pytest.mark.parametrize("change", [
    {"q": None}, {"q__data": None}, {"q__dtype": 2}, {"q__dtype": 7}, {"q__token_stride": -8}, {"q_heads": 0},
    {"q_heads": 2}, {"q_heads": 9}, {"q_heads": 1 << 20}, {"ws": ctypes.c_void_p((1 << 20) + 8)}])
def test_query_refusals(kv, change):
    refused(kv, ("attend", "select"), **change)


def test_attend_refusals(kv):
    refused(kv, ("attend",), o=None)
    refused(kv, ("attend",), o__dtype=1)  # another type than the queries
    refused(kv, ("attend",), keep=3)      # no list
    refused(kv, ("attend",), blocks=ctypes.c_void_p(1 << 20))
    refused(kv, ("attend",), blocks=ctypes.c_void_p(1 << 20), keep=-1)
    c = Call(kv)
    c.seqs.table_stride = c.seqs.table_width = 1 << 16
    c.seqs.longest = 1 << 22
    need = c.size(kv.OP_ATTEND)
    assert need > 0
    c.room = need - 1
    assert c.attend() == -1
    c.room, c.ws = need, None
    assert c.attend() == -1


@pytest.mark.parametrize("rows,call,heads", [("k", "read", 4), ("v", "read", 4), ("o", "attend", 8)])
def test_outputs_whose_elements_share_places(kv, rows, call, heads):
    wide, long = heads * 128, 30 * 128  # a token's heads, a head's tokens
    for token, head in ((0, 128), (wide, 0), (wide - 1, 128), (wide, 127), (128, long - 1), (127, long)):
        refused(kv, (call,), **{rows + "__token_stride": token, rows + "__head_stride": head})


def test_select_refusals(kv):
    for change in ({"keep": -1}, {"first": -1}, {"recent": 0}, {"first": 4}, {"recent": 5}, {"out": None},
                   {"q_heads": 4 * 129}, {"first": 1 << 62}, {"recent": 1 << 62}):
        refused(kv, ("select",), **change)
    # the scores of long sequences need a workspace
    c = Call(kv)
    c.keep = 4
    c.seqs.table_stride = c.seqs.table_width = 1 << 16
    c.seqs.longest = 1 << 22
    need = c.size(kv.OP_SELECT)
    assert need >= 30 * 4 * (1 << 16) * 4
    c.room = need - 1
    assert c.select() == -1
    c.room, c.ws = need, None
    assert c.select() == -1


def test_workspace_queries(kv):
    c = Call(kv)
    assert c.size(0) == 0 and c.size(3) == 0
    c.keep = -1
    assert c.size(kv.OP_ATTEND) == 0
    c.keep, c.cache.dim = 0, 80
    assert c.size(kv.OP_ATTEND) == 0 and c.size(kv.OP_SELECT) == 0


def test_python_refuses_host_tensors(kv):
    import torch
    with pytest.raises(TypeError):
        kv.new_cache(4, 2, 64, device="cpu")
    with pytest.raises(TypeError):
        kv.Seqs(torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))


def test_reference_codes():
    """The definition's own pins: every code is its own rounding, halfway goes to the even code,
    exponents are the least that hold."""
    for b in range(256):
        if b & 127 != 127:
            assert encode(E4M3_VALUES[b], 0) == b
    assert encode(0.5 * (E4M3_VALUES[8] + E4M3_VALUES[9]), 0) == 8
    assert encode(0.5 * (E4M3_VALUES[9] + E4M3_VALUES[10]), 0) == 10
    assert E4M3_VALUES[126] == 448 and E4M3_VALUES[1] == 2.0 ** -9
    for limit in (448.0, 127.0):
        for top in (1e-3, 0.5, 1.0, 3.5, 126.99, 127.0, 127.01, 448.0, 449.0, 896.0):
            e = least_exponent(top, limit)
            assert top <= limit * 2.0 ** e and top > limit * 2.0 ** (e - 1)
