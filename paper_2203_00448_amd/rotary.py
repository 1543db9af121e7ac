"""Python binding of rotary positions (mp_rotate of libmemoplan.so): argument marshalling only,
like kv.py, and the frequencies that a program makes once.

`rotate` turns pairs of elements of queries and keys by position * frequency, before they are written
to the cache and attended to.  It runs on `stream` (the current one of the queries' device if not given),
whichever device is current; tensors that are in use on another stream are the caller's to wait for.  It
builds no graph (tensors that require a gradient are refused where one is recorded): the gradient of a turn is the
inverse one, `rotate(..., inverse=True)`.
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import binding, kv
from .binding import MP_OK, PlanError
from .kv import _MOVED, _need, _rows

_lib = None


def load_library():
    """The library with this entry point declared."""
    global _lib
    if _lib is None:
        L = binding.load_library()
        p, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        L.mp_rotate.argtypes = [p, i64, p, i32, i32, ctypes.c_float, i32, i32, p, i32, p, p, i32, p, p]
        L.mp_rotate.restype = i32
        _lib = L
    return _lib


class Rotation:
    """What a program keeps of its rotary positions: the first `turned` elements of a head are turned, pair i
    by freq[i] radians a position, `base` ** (-2 i / turned) where nothing scales it.  pairs=False: elements
    (i, i + turned / 2) are a pair; True: (2 i, 2 i + 1).

    For contexts `factor` times longer than the `original` one, `scaling` is
      "linear": every frequency divided by factor;
      "base": the base times factor ** (turned / (turned - 2)), so that the slowest pair is divided by factor
         and the fastest is left;
      "blend": a pair that makes at least `high` turns in the original context is left, one that makes at
         most `low` divided by factor, linear in the turns between; results are multiplied by
         0.1 ln(factor) + 1, or `magnitude` if given.
    freq float64 [turned / 2] on the device replaces all of that."""

    SCALINGS = (None, "linear", "base", "blend")

    def __init__(self, turned: int, *, base: float = 10000.0, pairs: bool = False, scaling: str | None = None,
                 factor: float = 1.0, original: int = 4096, low: float = 1.0, high: float = 32.0,
                 magnitude: float | None = None, freq=None, device="cuda"):
        if turned < 2 or turned % 2:
            raise ValueError("turned must be even and at least 2")
        if scaling not in self.SCALINGS:
            raise ValueError(f"scaling must be one of {self.SCALINGS}")
        if not base > 0 or not factor > 0 or not high > low or not original > 0:
            raise ValueError("base, factor and original must be positive, high above low")
        if scaling == "base" and turned == 2:
            raise ValueError("one pair has no base")
        if freq is None:
            if scaling == "base":
                base = base * factor ** (turned / (turned - 2))
            made = []
            for i in range(turned // 2):
                f = base ** (-2.0 * i / turned)
                if scaling == "linear":
                    f /= factor
                elif scaling == "blend":
                    kept = min(1.0, max(0.0, (original * f / (2 * math.pi) - low) / (high - low)))
                    f *= kept + (1.0 - kept) / factor
                made.append(f)
            freq = torch.tensor(made, dtype=torch.float64, device=device)
        _need(freq, (torch.float64,), "freq", (turned // 2,))
        if not freq.is_contiguous():
            raise ValueError("freq must be contiguous")
        if magnitude is None:
            magnitude = 0.1 * math.log(factor) + 1.0 if scaling == "blend" else 1.0
        self.freq, self.turned, self.pairs, self.magnitude = freq, turned, bool(pairs), float(magnitude)
        self.device, self.index = freq.device, freq.get_device()
        self._freq, self._held = freq.data_ptr(), freq


def rotate(rotation: Rotation, position, q, k=None, *, out=None, k_out=None, inverse: bool = False, stream=None):
    """Turn q [tokens, q_heads, dim] and k [tokens, k_heads, dim] (bfloat16, float16 or float32, any strides over
    a contiguous last dimension) by position int32 [tokens] (mp_rotate).  `out` and `k_out` may be q and k.
    Returns out, or (out, k_out) with k."""
    if stream is not None or kv._device() != rotation.index:  # a launch would be the current device's
        with kv._current(rotation, stream):
            return rotate(rotation, position, q, k, out=out, k_out=k_out, inverse=inverse)
    L = load_library()
    if (q.requires_grad or (k is not None and k.requires_grad) or (out is not None and out.requires_grad)
            or (k_out is not None and k_out.requires_grad)) and torch.is_grad_enabled():
        raise ValueError("rotate builds no graph: call it under torch.no_grad(), and with inverse=True for the gradient")
    shape = q.shape
    if len(shape) != 3 or (k is not None and k.dim() != 3):
        raise ValueError("q and k must be [tokens, heads, dim]")
    if k is None and k_out is not None:
        raise ValueError("k_out needs k")
    index = rotation.index
    n, heads, dim = shape
    if not isinstance(position, torch.Tensor) or position.dtype is not torch.int32 or position.shape != (n,):
        _need(position, (torch.int32,), "position", (n,))
    if position.get_device() != index or not position.is_contiguous():
        raise ValueError("position must be contiguous and on the device of the rotation")
    dtypes = (q.dtype,)
    qa = _rows(q, "q", shape, _MOVED, index)
    if out is None:
        out = torch.empty(shape, dtype=q.dtype, device=q.device)
    oa = _rows(out, "out", shape, dtypes, index)
    ka = koa = None
    k_heads = 0
    if k is not None:
        k_heads = k.shape[1]
        shape = (n, k_heads, dim)
        ka = _rows(k, "k", shape, dtypes, index)
        if k_out is None:
            k_out = torch.empty(shape, dtype=k.dtype, device=k.device)
        koa = _rows(k_out, "k_out", shape, dtypes, index)
    at = ctypes.addressof
    rc = L.mp_rotate(position.data_ptr() or None, n, rotation._freq, rotation.turned, rotation.pairs,
                     rotation.magnitude, inverse, dim, at(qa), heads, at(oa), ka and at(ka), k_heads,
                     koa and at(koa), kv._stream(index))
    if rc != MP_OK:
        raise PlanError(rc, "rotary.rotate")
    return out if k is None else (out, k_out)
