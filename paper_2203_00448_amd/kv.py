"""Python binding of the key/value cache in 8 or 4 bits (mp_kv_* of libmemoplan.so):
argument marshalling only, like binding.py.

A program keeps a `Cache` (its memory), a `Seqs` for its batch (block table,
lengths, the call's rows), a status word and workspaces, and calls `write`,
`read`, `select` and `attend` on them; outputs may be views of a planned slab.
Each runs on `stream` (the current one of the cache's device if not given),
whichever device is current; tensors that are in use on another stream are the
caller's to wait for.  They are for serving: none has
a gradient, and an output shares no memory with an input.
The tensors that a handle was made of stay the caller's: changing their
values, not their places, changes what the next call sees.
"""
from __future__ import annotations

import contextlib
import ctypes

import torch

from . import binding
from .binding import PlanError, _finish, _p, new_status  # noqa: F401

E4M3, INT8, E2M1 = 0, 1, 4
OP_ATTEND, OP_SELECT = 1, 2
DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}

_i32, _i64, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p


class _CacheArg(ctypes.Structure):
    _fields_ = [("k_code", _vp), ("v_code", _vp), ("k_exp", _vp), ("v_exp", _vp),
                ("mean_code", _vp), ("mean_exp", _vp), ("n_blocks", _i64), ("heads", _i32),
                ("dim", _i32), ("block", _i32), ("kind", _i32)]


class _SeqsArg(ctypes.Structure):
    _fields_ = [("table", _vp), ("table_stride", _i64), ("table_width", _i64), ("length", _vp),
                ("begin", _vp), ("n_seqs", _i64), ("n_tokens", _i64), ("most_new", _i64),
                ("longest", _i64)]


class _RowsArg(ctypes.Structure):
    _fields_ = [("data", _vp), ("token_stride", _i64), ("head_stride", _i64), ("dtype", _i32)]


_lib = None


def load_library():
    """The library with the cache's entry points declared."""
    global _lib
    if _lib is None:
        L = binding.load_library()
        p, i32, i64, sz = _vp, _i32, _i64, ctypes.c_size_t
        L.mp_kv_write.argtypes = [p, p, p, p, p, p]
        L.mp_kv_write.restype = i32
        L.mp_kv_read.argtypes = [p, p, p, p, p, p]
        L.mp_kv_read.restype = i32
        L.mp_kv_attend.argtypes = [p, p, p, i32, ctypes.c_float, p, i64, p, p, p, sz, p, p]
        L.mp_kv_attend.restype = i32
        L.mp_kv_select.argtypes = [p, p, p, i32, i64, i64, i64, p, p, sz, p, p]
        L.mp_kv_select.restype = i32
        L.mp_kv_workspace_size.argtypes = [i32, p, p, i32, i64]
        L.mp_kv_workspace_size.restype = sz
        _lib = L
    return _lib


def _need(t, dtypes, name, shape=None):
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


class Cache:
    """Blocks of keys and values, all tensors contiguous and on one device.
    kind E4M3 or INT8: k_code uint8 [n_blocks, heads, block, dim], v_code uint8 [n_blocks, heads,
    dim, block], k_exp and v_exp int8 [n_blocks, heads], mean_code int8 [n_blocks, heads, dim],
    mean_exp int8 [n_blocks, heads].
    kind E2M1 (4 bits, a scale for each 32 dims of a token): k_code and v_code uint8 [n_blocks,
    heads, block, dim / 2], k_exp and v_exp uint8 [n_blocks, heads, dim / 32, block], exponents + 127;
    no means, so nothing is selected of it."""

    def __init__(self, k_code, v_code, k_exp, v_exp, mean_code=None, mean_exp=None, *, kind: int = E4M3):
        _need(k_code, (torch.uint8,), "k_code")
        if k_code.dim() != 4:
            raise ValueError("k_code must have 4 dimensions")
        if kind not in (E4M3, INT8, E2M1):
            raise ValueError("kind must be E4M3, INT8 or E2M1")
        n, h, t, d = k_code.shape
        if kind == E2M1:
            _need(v_code, (torch.uint8,), "v_code", (n, h, t, d))
            d *= 2
            for x, name in ((k_exp, "k_exp"), (v_exp, "v_exp")):
                _need(x, (torch.uint8,), name, (n, h, d // 32, t))
            if mean_code is not None or mean_exp is not None:
                raise ValueError("a cache in 4 bits has no means")
            self.tensors = (k_code, v_code, k_exp, v_exp)
        else:
            _need(v_code, (torch.uint8,), "v_code", (n, h, d, t))
            for x, name in ((k_exp, "k_exp"), (v_exp, "v_exp"), (mean_exp, "mean_exp")):
                _need(x, (torch.int8,), name, (n, h))
            _need(mean_code, (torch.int8,), "mean_code", (n, h, d))
            self.tensors = (k_code, v_code, k_exp, v_exp, mean_code, mean_exp)
        for x in self.tensors:
            if not x.is_contiguous() or x.device != k_code.device:
                raise ValueError("a cache's tensors must be contiguous and on one device")
        self.k_code, self.v_code, self.k_exp, self.v_exp = self.tensors[:4]
        self.mean_code, self.mean_exp = mean_code, mean_exp
        self.n_blocks, self.heads, self.block, self.dim, self.kind = n, h, t, d, kind
        self.device, self.index = k_code.device, k_code.get_device()
        at = [x.data_ptr() for x in self.tensors] + [None] * (6 - len(self.tensors))
        self._arg = _CacheArg(*at, n, h, d, t, kind)
        self._ref = ctypes.addressof(self._arg)

    @property
    def nbytes(self) -> int:
        return sum(x.numel() for x in self.tensors)


def new_cache(n_blocks: int, heads: int, dim: int, *, block: int = 64, kind: int = E4M3,
              device="cuda") -> Cache:
    """A cache of zeros."""
    def z(*shape, dtype=torch.int8):
        return torch.zeros(shape, dtype=dtype, device=device)

    if kind == E2M1:
        codes, exps = (n_blocks, heads, block, dim // 2), (n_blocks, heads, dim // 32, block)
        return Cache(*(torch.zeros(codes, dtype=torch.uint8, device=device) for _ in range(2)),
                     *(torch.full(exps, 127, dtype=torch.uint8, device=device) for _ in range(2)), kind=kind)
    return Cache(z(n_blocks, heads, block, dim, dtype=torch.uint8),
                 z(n_blocks, heads, dim, block, dtype=torch.uint8), z(n_blocks, heads),
                 z(n_blocks, heads), z(n_blocks, heads, dim), z(n_blocks, heads), kind=kind)


class Seqs:
    """The sequences of a call: table int32 [n_seqs, width] (rows may be strided), length int32
    [n_seqs] (the call's tokens included), begin int64 [n_seqs + 1] or None (one row for each
    sequence).  `tokens` rows in all, at most `most_new` of a sequence, no sequence longer than
    `longest`; what is not given is the most that the shapes allow (`tokens` is read from begin,
    which waits for the device)."""

    def __init__(self, table, length, *, begin=None, tokens: int | None = None,
                 most_new: int | None = None, longest: int | None = None):
        _need(length, (torch.int32,), "length")
        n = length.numel()
        _need(table, (torch.int32,), "table")
        if table.dim() != 2 or table.shape[0] != n:
            raise ValueError("table must be [n_seqs, width]")
        if table.shape[1] > 1 and table.stride(1) != 1:
            raise ValueError("a row of table must be contiguous")
        if n > 1 and table.stride(0) < table.shape[1]:
            raise ValueError("rows of table must not share places")
        if length.dim() != 1 or not length.is_contiguous():
            raise ValueError("length must be a contiguous vector")
        if table.device != length.device:
            raise ValueError("table and length must be on one device")
        if begin is not None:
            _need(begin, (torch.int64,), "begin", (n + 1,))
            if not begin.is_contiguous() or begin.device != length.device:
                raise ValueError("begin must be contiguous and on the device of length")
            if tokens is None:
                tokens = int(begin[-1].item())
        elif tokens is None:
            tokens = n
        elif tokens != n:
            raise ValueError("without begin there is one row for each sequence")
        self.table, self.length, self.begin = table, length, begin
        self.n_seqs, self.tokens = n, int(tokens)
        self.most_new = int(most_new) if most_new is not None else self.tokens if begin is not None else 1
        self.longest, self.device = longest, length.device
        width = table.shape[1]
        self._fields = (table.data_ptr() or None, max(width, table.stride(0)), width, length.data_ptr() or None,
                        begin.data_ptr() if begin is not None else None, n, self.tokens, self.most_new)
        self._last = (None, None)

    def _for(self, cache: Cache):
        """Its argument, with the bound on the lengths, for a cache's blocks.  One that was handed out never
        changes (another thread's call may be reading it): the caller holds it during its call."""
        if cache.device != self.device:
            raise ValueError("cache and sequences must be on one device")
        longest = self._fields[2] * cache.block if self.longest is None else self.longest
        last = self._last
        if last[0] != longest:
            last = self._last = (longest, _SeqsArg(*self._fields, longest))
        return last[1]


_MOVED = (torch.bfloat16, torch.float16, torch.float32)
_QUERIES = (torch.bfloat16, torch.float16)


def _rows(t, name, shape, dtypes, index):
    """A tensor's rows as an argument.  These calls are short beside what a launch costs, so their
    checks look at each property once."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in dtypes or t.shape != shape:
        _need(t, dtypes, name, shape)
    if t.get_device() != index:
        raise ValueError(f"{name} must be on the device of the cache")
    strides = t.stride()
    if strides[2] != 1:
        raise ValueError(f"{name} must be contiguous in its last dimension")
    return _RowsArg(t.data_ptr(), strides[0], strides[1], DTYPES[t.dtype])


_stream, _device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


@contextlib.contextmanager
def _current(cache, stream):
    """The cache's device and `stream`, if given, current for a call: what it allocates is theirs, and so
    is the wait of check."""
    if stream is not None and stream.device != cache.device:
        raise ValueError("stream must be of the device of the cache")
    with torch.cuda.device(cache.device), torch.cuda.stream(stream):
        yield


def _word(status, cache):
    if status is None:
        return new_status(cache.device)
    if not status.is_cuda or status.dtype is not torch.int32:
        _need(status, (torch.int32,), "status")
    if status.numel() != 1 or status.get_device() != cache.index:
        raise ValueError("status must be one word on the device of the cache")
    return status


def workspace_size(op: int, cache: Cache, seqs: Seqs, *, q_heads: int, keep: int = 0) -> int:
    """mp_kv_workspace_size: bytes of workspace of attend (`keep` 0 without blocks) or select."""
    held = seqs._for(cache)
    return int(load_library().mp_kv_workspace_size(op, cache._ref, ctypes.addressof(held), q_heads, keep))


def workspace(op: int, cache: Cache, seqs: Seqs, *, q_heads: int, keep: int = 0):
    """A new workspace of that size."""
    need = workspace_size(op, cache, seqs, q_heads=q_heads, keep=keep)
    return torch.empty(max(need, 16), dtype=torch.uint8, device=cache.device)


def write(cache: Cache, seqs: Seqs, k, v, *, status=None, check: bool = True, stream=None):
    """Store the call's keys and values (mp_kv_write): k, v [tokens, heads, dim] in bfloat16,
    float16 or float32, any strides over a contiguous last dimension."""
    if stream is not None or _device() != cache.index:  # a launch would be the current device's
        with _current(cache, stream):
            return write(cache, seqs, k, v, status=status, check=check)
    L = load_library()
    shape = (seqs.tokens, cache.heads, cache.dim)
    ka, va = _rows(k, "k", shape, _MOVED, cache.index), _rows(v, "v", shape, _MOVED, cache.index)
    status = _word(status, cache)
    held = seqs._for(cache)
    rc = L.mp_kv_write(cache._ref, ctypes.addressof(held), ctypes.addressof(ka), ctypes.addressof(va),
                       status.data_ptr(), _stream(cache.index))
    _finish(rc, status, "kv.write", check)


def read(cache: Cache, seqs: Seqs, *, dtype=torch.bfloat16, out=None, status=None,
         check: bool = True, stream=None):
    """Read back the call's tokens (mp_kv_read): (k, v) [tokens, heads, dim]."""
    if stream is not None or _device() != cache.index:  # a launch would be the current device's
        with _current(cache, stream):
            return read(cache, seqs, dtype=dtype, out=out, status=status, check=check)
    L = load_library()
    shape = (seqs.tokens, cache.heads, cache.dim)
    if out is None:
        out = tuple(torch.empty(shape, dtype=dtype, device=cache.device) for _ in range(2))
    k, v = out
    ka, va = _rows(k, "k", shape, _MOVED, cache.index), _rows(v, "v", shape, _MOVED, cache.index)
    status = _word(status, cache)
    held = seqs._for(cache)
    rc = L.mp_kv_read(cache._ref, ctypes.addressof(held), ctypes.addressof(ka), ctypes.addressof(va),
                      status.data_ptr(), _stream(cache.index))
    _finish(rc, status, "kv.read", check)
    return k, v


def _space(op, cache, seqs, q_heads, keep, workspace):
    if workspace is None:
        workspace = globals()["workspace"](op, cache, seqs, q_heads=q_heads, keep=keep)
    elif not workspace.is_cuda:
        raise TypeError("workspace must be a CUDA (HIP) tensor")
    elif not workspace.is_contiguous() or workspace.get_device() != cache.index:
        raise ValueError("workspace must be contiguous and on the device of the cache")
    return workspace.data_ptr(), workspace.nbytes, workspace


def attend(cache: Cache, seqs: Seqs, q, *, scale: float | None = None, blocks=None, out=None,
           lse=None, status=None, workspace=None, check: bool = True, stream=None):
    """Attention of q [tokens, q_heads, dim] (bfloat16 or float16) over the cache
    (mp_kv_attend), causal: the rows of a sequence are its last tokens.  `scale` defaults to
    dim ** -0.5.  `blocks` int32 [tokens, heads, keep] limits each row to these of its
    sequence's blocks.  `lse` float32 [tokens, q_heads], if given, gets the logarithms of the
    sums.  Returns out."""
    if stream is not None or _device() != cache.index:  # a launch would be the current device's
        with _current(cache, stream):
            return attend(cache, seqs, q, scale=scale, blocks=blocks, out=out, lse=lse, status=status,
                          workspace=workspace, check=check)
    L = load_library()
    if q.dim() != 3:
        raise ValueError("q must be [tokens, q_heads, dim]")
    heads = q.shape[1]
    rows = (seqs.tokens, heads, cache.dim)
    qa = _rows(q, "q", rows, _QUERIES, cache.index)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    oa = _rows(out, "out", rows, (q.dtype,), cache.index)
    keep, named = 0, None
    if blocks is not None:
        _need(blocks, (torch.int32,), "blocks")
        if blocks.dim() != 3 or blocks.shape[:2] != (seqs.tokens, cache.heads) or not blocks.is_contiguous():
            raise ValueError("blocks must be a contiguous [tokens, heads, keep]")
        if blocks.shape[2] < 1 or blocks.get_device() != cache.index:
            raise ValueError("blocks must name at least one place and be on the device of the cache")
        keep, named = blocks.shape[2], blocks.data_ptr()
    if lse is not None:
        _need(lse, (torch.float32,), "lse", (seqs.tokens, heads))
        if not lse.is_contiguous() or lse.get_device() != cache.index:
            raise ValueError("lse must be contiguous and on the device of the cache")
    space, have, _held = _space(OP_ATTEND, cache, seqs, heads, keep, workspace)
    status = _word(status, cache)
    held = seqs._for(cache)
    rc = L.mp_kv_attend(cache._ref, ctypes.addressof(held), ctypes.addressof(qa), heads,
                        cache.dim ** -0.5 if scale is None else scale, named, keep,
                        ctypes.addressof(oa), lse.data_ptr() if lse is not None else None,
                        space, have, status.data_ptr(), _stream(cache.index))
    _finish(rc, status, "kv.attend", check)
    return out


def select(cache: Cache, seqs: Seqs, q, *, keep: int, first: int = 1, recent: int = 1, out=None,
           status=None, workspace=None, check: bool = True, stream=None):
    """The blocks of each row and key head that attend is to read (mp_kv_select): the first
    `first`, the last `recent` and the best-scored others, `keep` in all, int32 [tokens, heads,
    keep], ascending, -1 beyond the last."""
    if stream is not None or _device() != cache.index:  # a launch would be the current device's
        with _current(cache, stream):
            return select(cache, seqs, q, keep=keep, first=first, recent=recent, out=out, status=status,
                          workspace=workspace, check=check)
    L = load_library()
    if q.dim() != 3:
        raise ValueError("q must be [tokens, q_heads, dim]")
    heads = q.shape[1]
    rows = (seqs.tokens, heads, cache.dim)
    qa = _rows(q, "q", rows, _QUERIES, cache.index)
    shape = (seqs.tokens, cache.heads, int(keep))
    if out is None:
        out = torch.empty(shape, dtype=torch.int32, device=q.device)
    _need(out, (torch.int32,), "out", shape)
    if not out.is_contiguous() or out.get_device() != cache.index:
        raise ValueError("out must be contiguous and on the device of the cache")
    space, have, _held = _space(OP_SELECT, cache, seqs, heads, keep, workspace)
    status = _word(status, cache)
    held = seqs._for(cache)
    rc = L.mp_kv_select(cache._ref, ctypes.addressof(held), ctypes.addressof(qa), heads, keep, first, recent,
                        out.data_ptr() or None, space, have, status.data_ptr(),
                        _stream(cache.index))
    _finish(rc, status, "kv.select", check)
    return out
