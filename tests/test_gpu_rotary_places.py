"""Rotary positions written to the places that they are read from, by tensors of other strides."""
import pytest
import torch

from gpu_util import dev
from test_gpu_rotary import BF16, F16, F32, module, near, positions

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("n,heads,key_heads", [(1, 5, 2), (9, 1, 1), (1, 1, 0), (1, 3, 1), (4, 1, 3)])
@pytest.mark.parametrize("dim,turned", [(66, 66), (70, 62), (1030, 1030), (2062, 1550), (4094, 4094)])
def test_strides_of_an_axis_of_one(dim, turned, n, heads, key_heads, pairs, dtype):
    """In place where the output names other strides of axes that have one place: the same bits as apart.  Heads whose
    pieces of 16 bytes are no whole ones and more than a wave's."""
    rotary = module()
    r = rotary.Rotation(turned, pairs=pairs)
    p = positions(n, 3000)
    at = dev(p, torch.int32)
    rows = torch.randn(n, heads + key_heads, dim + 2, device="cuda").to(dtype)
    before = rows.clone()

    def parts(of):
        return of[:, :heads, :dim], of[:, heads:, :dim] if key_heads else None

    def elsewise(x):
        """The same places, by other strides of what has one place."""
        n, h, d = x.shape
        return x.as_strided((n, h, d), (7 * dim if n == 1 else x.stride(0), 5 * dim if h == 1 else x.stride(1), 1))

    q, k = parts(rows)
    apart = rotary.rotate(r, at, q, k)
    apart = apart if key_heads else (apart, None)
    assert torch.equal(rows, before)
    rotary.rotate(r, at, q, k, out=elsewise(q), k_out=elsewise(k) if key_heads else None)
    assert torch.equal(q, apart[0])
    near(q, parts(before)[0], p, r)
    if key_heads:
        assert torch.equal(k, apart[1])
    assert torch.equal(rows[..., dim:], before[..., dim:])
