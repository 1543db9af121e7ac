"""Python binding of the blocks given to requests (mp_kv_extend, mp_kv_release of
libmemoplan.so): argument marshalling only, like kv.py.

A program keeps a `Pool` (block ids, and how many of them are taken), its block table, its
lengths, a `Step` (what the calls of a step read), a status word and a workspace.  `release` takes
back the blocks of requests that ended, `extend` gives blocks to the new tokens of the others and
makes the step's lengths, row bounds, positions and slots; nothing waits for the host, so both
can be recorded in a graph.  Each runs on `stream` (the current one of the pool's device if not
given), whichever device is current; tensors that are in use on another stream are the caller's to
wait for.  Outputs are written in place: `length` and the pool's counter too, if no others are given.
The tensors that a handle was made of stay the caller's: changing their values, not their places, changes
what the next call sees, and another tensor in an attribute's place does not.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding, kv
from .binding import MP_OK, _finish, new_status  # noqa: F401
from .kv import _need

_lib = None


def load_library():
    """The library with these entry points declared."""
    global _lib
    if _lib is None:
        L = binding.load_library()
        p, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        L.mp_kv_extend.argtypes = [p, i64, p, p, i64, i64, i32, p, p, i64, i64, p, p, p, p, p, p, sz, p, p]
        L.mp_kv_extend.restype = i32
        L.mp_kv_release.argtypes = [p, i64, p, p, i64, i64, i32, p, p, i64, p, p, p, sz, p, p]
        L.mp_kv_release.restype = i32
        L.mp_kv_pages_workspace_size.argtypes = [i64]
        L.mp_kv_pages_workspace_size.restype = sz
        _lib = L
    return _lib


def _vector(t, dtype, name, n, index):
    """A vector's address.  These calls are short beside what a launch costs, so their checks look at each
    property once."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.dim() != 1 or t.numel() != n or not t.is_cuda:
        _need(t, (dtype,), name, (n,))
    if t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous and on one device with the others")
    return t.data_ptr() or None


class Pool:
    """Block ids int32 [n] and how many blocks are taken, int64 [1]: ids[used:] are free and given out in order,
    what lies before them means nothing once a block came back.  Two handles may share `ids`."""

    def __init__(self, ids, used):
        _need(ids, (torch.int32,), "ids")
        _need(used, (torch.int64,), "used", (1,))
        if ids.dim() != 1 or not ids.is_contiguous() or used.device != ids.device:
            raise ValueError("ids must be a contiguous vector, on the device of used")
        self.ids, self.used = ids, used
        self.device, self.index = ids.device, ids.get_device()
        self._at, self._held = (ids.data_ptr() or None, ids.numel(), used.data_ptr()), (ids, used)


def new_pool(n_blocks: int, *, device="cuda") -> Pool:
    """Blocks 0 to n_blocks - 1, all free."""
    return Pool(torch.arange(n_blocks, dtype=torch.int32, device=device),
                torch.zeros(1, dtype=torch.int64, device=device))


class Step:
    """What the calls of a step read: length int32 [n_seqs], begin int64 [n_seqs + 1], position int32
    [tokens], slot int64 [tokens].  `length` is where the last `extend` with this handle put the lengths: in place
    where no length_out was given, so the first tensor is filled only as a call's length_out."""

    def __init__(self, length, begin, position, slot):
        self.length, self.begin, self.position, self.slot = length, begin, position, slot
        n, room, self.index = length.numel(), slot.numel(), begin.get_device()
        _vector(length, torch.int32, "length", n, self.index)
        self._at = (_vector(begin, torch.int64, "begin", n + 1, self.index),
                    _vector(position, torch.int32, "position", room, self.index),
                    _vector(slot, torch.int64, "slot", room, self.index), room, n)
        self._held = (begin, position, slot)


def new_step(n_seqs: int, tokens: int, *, device="cuda") -> Step:
    """A step of at most `tokens` new tokens."""
    def z(n, dtype):
        return torch.zeros(n, dtype=dtype, device=device)

    return Step(z(n_seqs, torch.int32), z(n_seqs + 1, torch.int64), z(tokens, torch.int32), z(tokens, torch.int64))


def workspace(n_seqs: int, *, device="cuda"):
    """A new workspace of mp_kv_pages_workspace_size bytes."""
    return torch.empty(int(load_library().mp_kv_pages_workspace_size(n_seqs)), dtype=torch.uint8, device=device)


def _space(n, workspace, pool):
    if workspace is None:
        workspace = globals()["workspace"](n, device=pool.device)
    elif not workspace.is_cuda:
        raise TypeError("workspace must be a CUDA (HIP) tensor")
    elif workspace.get_device() != pool.index or not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous and on the device of the pool")
    return workspace


def _table(table, n, index):
    if not isinstance(table, torch.Tensor) or table.dtype is not torch.int32 or not table.is_cuda:
        _need(table, (torch.int32,), "table")
    shape = table.shape
    if len(shape) != 2 or shape[0] != n or table.get_device() != index:
        raise ValueError("table must be [n_seqs, width], on the device of the pool")
    width, (stride, step) = shape[1], table.stride()
    if width > 1 and step != 1:
        raise ValueError("a row of table must be contiguous")
    if n > 1 and stride < width:
        raise ValueError("rows of table must not share places")
    return table.data_ptr() or None, max(width, stride), width


def extend(pool: Pool, table, length, more, *, block: int = 64, step: Step, length_out=None, used_out=None,
           status=None, workspace=None, check: bool = True, stream=None) -> Step:
    """Give blocks to more int32 [n_seqs] new tokens of sequences that hold `length` int32 [n_seqs]
    (mp_kv_extend): entries of table int32 [n_seqs, width] and the pool's counter are written in place, the lengths
    to length_out (`length` if not given), which is step.length from then on, the rest to `step`, which is
    returned."""
    if stream is not None or kv._device() != pool.index:  # a launch would be the current device's
        with kv._current(pool, stream):
            return extend(pool, table, length, more, block=block, step=step, length_out=length_out,
                          used_out=used_out, status=status, workspace=workspace, check=check)
    L = load_library()
    n, index = length.numel(), pool.index
    t, t_stride, width = _table(table, n, index)
    lengths = _vector(length, torch.int32, "length", n, index)
    new = _vector(more, torch.int32, "more", n, index)
    out = lengths if length_out is None else _vector(length_out, torch.int32, "length_out", n, index)
    ids, n_ids, used = pool._at
    used_to = used if used_out is None else _vector(used_out, torch.int64, "used_out", 1, index)
    begin, position, slot, room, of = step._at
    if of != n or step.index != index:
        raise ValueError("step must be of as many sequences and on the device of the pool")
    space = _space(n, workspace, pool)
    status = kv._word(status, pool)
    rc = L.mp_kv_extend(ids, n_ids, used, t, t_stride, width, block, lengths, new, n, room, out, used_to, begin,
                        position, slot, space.data_ptr(), space.nbytes, status.data_ptr(), kv._stream(index))
    if rc == MP_OK:
        step.length = length if length_out is None else length_out
    _finish(rc, status, "pages.extend", check)
    return step


def release(pool: Pool, table, length, done, *, block: int = 64, length_out=None, used_out=None, status=None,
            workspace=None, check: bool = True, stream=None):
    """Take back the blocks of the sequences with done bool or uint8 [n_seqs] set (mp_kv_release): the pool's
    ids and counter are written in place, the lengths (0 for these) to length_out, `length` if not given.
    Returns length_out."""
    if stream is not None or kv._device() != pool.index:  # a launch would be the current device's
        with kv._current(pool, stream):
            return release(pool, table, length, done, block=block, length_out=length_out, used_out=used_out,
                           status=status, workspace=workspace, check=check)
    L = load_library()
    n, index = length.numel(), pool.index
    t, t_stride, width = _table(table, n, index)
    lengths = _vector(length, torch.int32, "length", n, index)
    if done.dtype is torch.uint8:
        ended = _vector(done, torch.uint8, "done", n, index)
    else:
        ended = _vector(done, torch.bool, "done", n, index)
    out = lengths if length_out is None else _vector(length_out, torch.int32, "length_out", n, index)
    ids, n_ids, used = pool._at
    used_to = used if used_out is None else _vector(used_out, torch.int64, "used_out", 1, index)
    space = _space(n, workspace, pool)
    status = kv._word(status, pool)
    rc = L.mp_kv_release(ids, n_ids, used, t, t_stride, width, block, lengths, ended, n, out, used_to,
                         space.data_ptr(), space.nbytes, status.data_ptr(), kv._stream(index))
    _finish(rc, status, "pages.release", check)
    return length if length_out is None else length_out
