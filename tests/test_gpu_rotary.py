"""Rotary positions on the GPU against their definition in 64 bits, and against differences."""
import math

import numpy as np
import pytest
import torch

from gpu_util import dev, host, need_gpu

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
HALF_STEP = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}
LEAST_STEP = {BF16: 2.0 ** -134, F16: 2.0 ** -25, F32: 2.0 ** -150}


def module():
    need_gpu()
    from paper_2203_00448_amd import rotary
    return rotary


def reference(x, position, freq, magnitude, turned, pairs, inverse):
    """(turned x, |a| + |b| of each element's pair times magnitude) in 64 bits."""
    angle = position.astype(np.float64)[:, None, None] * freq * (-1.0 if inverse else 1.0)
    c, s = np.cos(angle) * magnitude, np.sin(angle) * magnitude
    y, size = x.copy(), np.zeros_like(x)
    a, b = (slice(0, turned, 2), slice(1, turned, 2)) if pairs else (slice(0, turned // 2), slice(turned // 2, turned))
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    size[..., a] = size[..., b] = (np.abs(x[..., a]) + np.abs(x[..., b])) * abs(magnitude)
    return y, size


def near(got, x, position, rotation, inverse=False):
    """A sine or cosine is off by 2^-22 at most (the angle below an eighth of a turn, its series and the
    magnitude are each rounded to 24 bits, some of them twice), two products and a sum by 2^-24 each; the
    result is rounded once.  Elements that are not turned are the same bits."""
    x, dtype = host(x.double()), got.dtype
    want, size = reference(x, position, host(rotation.freq), rotation.magnitude, rotation.turned, rotation.pairs, inverse)
    got = host(got.double())
    bound = HALF_STEP[dtype] * np.abs(want) + (2.0 ** -22 + 3 * 2.0 ** -24) * 1.01 * size + LEAST_STEP[dtype]
    off = np.abs(got - want)
    assert np.all(off <= bound), (off / bound).max()
    assert np.array_equal(got[..., rotation.turned:], x[..., rotation.turned:])


def positions(n, far, seed=0):
    p = np.random.default_rng(seed).integers(0, far, n)
    p[0] = 0
    p[-1] = far - 1
    return p


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("n,heads,key_heads,dim,turned", [
    (1, 1, 0, 64, 64), (1, 32, 8, 128, 128), (64, 32, 8, 128, 128), (5, 3, 1, 80, 80), (7, 5, 2, 96, 32), (3, 2, 3, 66, 66),
    (4, 7, 1, 128, 2), (2, 1, 1, 2, 2), (300, 8, 1, 192, 64), (9, 4, 4, 256, 250), (3000, 2, 1, 128, 128),
    (6000, 12, 4, 48, 16), (5, 2, 1, 4096, 4096), (2, 300, 5, 64, 64)])
def test_rotate(n, heads, key_heads, dim, turned, pairs, dtype):
    rotary = module()
    r = rotary.Rotation(turned, pairs=pairs)
    gen = torch.Generator(device="cuda").manual_seed(n + dim)
    q = torch.randn(n, heads, dim, generator=gen, device="cuda").to(dtype)
    k = torch.randn(n, key_heads, dim, generator=gen, device="cuda").to(dtype) if key_heads else None
    p = positions(n, 5000)
    for inverse in (False, True):
        got = rotary.rotate(r, dev(p, torch.int32), q, k, inverse=inverse)
        if k is None:
            near(got, q, p, r, inverse)
        else:
            near(got[0], q, p, r, inverse)
            near(got[1], k, p, r, inverse)


@pytest.mark.parametrize("pairs", [False, True])
def test_far_positions(pairs):
    """Angles of 2^31 radians: half a place of theirs in 64 bits is 2^-23, the same in the definition."""
    rotary = module()
    r = rotary.Rotation(128, pairs=pairs, base=500000.0)
    q = torch.randn(200, 4, 128, device="cuda")
    p = positions(200, 2 ** 31 - 1)
    near(rotary.rotate(r, dev(p, torch.int32), q), q, p, r)
    p = -p
    near(rotary.rotate(r, dev(p, torch.int32), q), q, p, r)


def test_every_quarter():
    """Angles at and around whole eighths of a turn."""
    rotary = module()
    freq = torch.tensor([math.pi / 4, math.pi / 4 + 1e-9, math.pi / 2, math.pi - 1e-7], dtype=torch.float64, device="cuda")
    r = rotary.Rotation(8, freq=freq)
    p = np.arange(-40, 40)
    q = torch.randn(80, 1, 8, device="cuda")
    near(rotary.rotate(r, dev(p, torch.int32), q), q, p, r)


@pytest.mark.parametrize("scaling", [None, "linear", "base", "blend"])
def test_scaled_frequencies(scaling):
    rotary = module()
    r = rotary.Rotation(64, base=10000.0, scaling=scaling, factor=8.0, original=2048, low=1.0, high=32.0)
    i = np.arange(32)
    plain = 10000.0 ** (-i / 32)
    if scaling == "blend":
        turns = 2048 * plain / (2 * math.pi)
        kept = np.clip((turns - 1) / 31, 0, 1)
        want, magnitude = plain * kept + plain / 8 * (1 - kept), 0.1 * math.log(8.0) + 1
        assert kept[0] == 1 and kept[-1] == 0
    else:
        want = {None: plain, "linear": plain / 8, "base": (10000.0 * 8 ** (64 / 62)) ** (-i / 32)}[scaling]
        magnitude = 1.0
    assert np.allclose(host(r.freq), want, rtol=1e-13, atol=0) and abs(r.magnitude - magnitude) < 1e-15
    if scaling == "base":
        assert abs(float(r.freq[-1]) * 8 / plain[-1] - 1) < 1e-12  # the slowest pair: divided by factor
    q = torch.randn(50, 2, 64, device="cuda").to(BF16)
    p = positions(50, 16384)
    near(rotary.rotate(r, dev(p, torch.int32), q), q, p, r)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("shift", [0, 1, 2, 4])  # of elements: 2 to 16 bytes at a time
def test_in_place_and_strided(shift, pairs, dtype):
    """Queries and keys side by side in wider rows, turned where they are; the rest of the rows is left."""
    rotary = module()
    r = rotary.Rotation(64, pairs=pairs)
    rows = torch.randn(30, 12, 96 + 8, device="cuda").to(dtype)
    before = rows.clone()
    q, k = rows[:, :7, shift:96 + shift], rows[:, 8:11, shift:96 + shift]
    p = positions(30, 999)
    q0, k0 = q.clone(), k.clone()
    apart = rotary.rotate(r, dev(p, torch.int32), q, k)
    assert torch.equal(rows, before)
    got = rotary.rotate(r, dev(p, torch.int32), q, k, out=q, k_out=k)
    assert got[0] is q and torch.equal(q, apart[0]) and torch.equal(k, apart[1])
    near(q, q0, p, r)
    near(k, k0, p, r)
    rows[:, :7, shift:96 + shift], rows[:, 8:11, shift:96 + shift] = q0, k0
    assert torch.equal(rows, before)
    # heads outside tokens, one row for all heads
    t = torch.randn(4, 30, 96, device="cuda").to(dtype).transpose(0, 1)
    near(rotary.rotate(r, dev(p, torch.int32), t), t, p, r)
    same = torch.randn(30, 1, 96, device="cuda").to(dtype).expand(30, 5, 96)
    near(rotary.rotate(r, dev(p, torch.int32), same), same, p, r)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dim,turned", [(66, 66), (66, 6), (96, 76), (70, 62), (128, 50), (41, 34), (16, 2), (192, 134),
                                        (256, 74), (25, 18)])
def test_no_whole_pieces(dim, turned, pairs, dtype):
    """Heads and turned elements that are no multiples of 16 bytes: out of place, in place, and one of the two; what
    lies between the heads is left."""
    rotary = module()
    r = rotary.Rotation(turned, pairs=pairs)
    rows = torch.randn(37, 9, dim + 3, device="cuda").to(dtype)
    q, k = rows[:, :5, 1:dim + 1], rows[:, 6:9, 1:dim + 1]
    p = positions(37, 5000)
    at, q0, k0, before = dev(p, torch.int32), q.clone(), k.clone(), rows.clone()
    wide = torch.full((37, 9, dim + 3), 7.0, device="cuda").to(dtype)
    apart = rotary.rotate(r, at, q, k, out=wide[:, :5, 2:dim + 2], k_out=wide[:, 6:9, 2:dim + 2])
    assert torch.equal(rows, before) and bool((wide[:, 5] == 7).all())
    assert bool((wide[:, :, :2] == 7).all()) and bool((wide[:, :, dim + 2:] == 7).all())
    near(apart[0], q0, p, r)
    near(apart[1], k0, p, r)
    k_out = torch.empty_like(k0)
    rotary.rotate(r, at, q, k, out=q, k_out=k_out)
    assert torch.equal(q, apart[0]) and torch.equal(k_out, apart[1]) and torch.equal(k, k0)
    q.copy_(q0)
    rotary.rotate(r, at, q, k, out=q, k_out=k)
    assert torch.equal(q, apart[0]) and torch.equal(k, apart[1])
    q.copy_(q0), k.copy_(k0)
    assert torch.equal(rows, before)


@pytest.mark.parametrize("pairs", [False, True])
def test_gradient(pairs):
    """The inverse turn is the gradient: against differences of the definition, and <turn x, y> = <x, inverse y>."""
    rotary = module()
    r = rotary.Rotation(12, pairs=pairs, scaling="blend", factor=4.0, original=64)
    p = positions(6, 300)
    x = torch.randn(6, 2, 16, dtype=torch.float64, device="cuda")
    y = torch.randn(6, 2, 16, device="cuda")
    grad = host(rotary.rotate(r, dev(p, torch.int32), y, inverse=True).double())
    f = lambda z: float((reference(z, p, host(r.freq), r.magnitude, 12, pairs, False)[0] * host(y.double())).sum())  # noqa: E731
    x0 = host(x)
    for at in [(0, 0, 0), (1, 1, 3), (5, 0, 11), (3, 1, 15), (2, 0, 6)]:
        up, down = x0.copy(), x0.copy()
        up[at] += 0.5
        down[at] -= 0.5  # the turn is linear: differences have no error but rounding
        assert abs(f(up) - f(down) - grad[at]) < 1e-6 * 12
    z = torch.randn(6, 2, 16, device="cuda")
    turned = rotary.rotate(r, dev(p, torch.int32), z)
    left, right = float((turned.double() * y.double()).sum()), float((z.double() * torch.from_numpy(grad).cuda()).sum())
    assert abs(left - right) < 192 * 8 * 2.0 ** -21


def test_large_values():
    rotary = module()
    r = rotary.Rotation(64)
    p = positions(20, 4000)
    for dtype, size in ((BF16, 2.0 ** 120), (F32, 2.0 ** 120), (F16, 2.0 ** 12), (F32, 2.0 ** -120)):
        q = (torch.randn(20, 3, 64, device="cuda") * size).to(dtype)
        near(rotary.rotate(r, dev(p, torch.int32), q), q, p, r)


def test_empty_and_other_stream():
    rotary = module()
    r = rotary.Rotation(64)
    none = torch.zeros(0, 4, 64, device="cuda")
    assert rotary.rotate(r, torch.zeros(0, dtype=torch.int32, device="cuda"), none).shape == (0, 4, 64)
    q, p = torch.randn(100, 4, 64, device="cuda"), positions(100, 500)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(q)
    rotary.rotate(r, dev(p, torch.int32), q, out=out, stream=side)
    side.synchronize()
    near(out, q, p, r)


def test_refusals():
    rotary = module()
    from paper_2203_00448_amd import binding
    for bad in ({"turned": 7}, {"turned": 0}, {"turned": 64, "scaling": "other"}, {"turned": 64, "base": 0.0},
                {"turned": 64, "factor": -1.0}, {"turned": 2, "scaling": "base", "factor": 2.0},
                {"turned": 64, "low": 4.0, "high": 4.0}):
        with pytest.raises(ValueError):
            rotary.Rotation(**bad)
    with pytest.raises(TypeError):
        rotary.Rotation(8, freq=torch.ones(4, device="cuda"))
    r = rotary.Rotation(64)
    p = torch.zeros(5, dtype=torch.int32, device="cuda")
    q = torch.zeros(5, 2, 64, device="cuda")
    with pytest.raises(binding.PlanError):
        rotary.rotate(r, p, q[..., :32])
    with pytest.raises(ValueError):
        rotary.rotate(r, p[:4], q)
    with pytest.raises(TypeError):
        rotary.rotate(r, p.long(), q)
    with pytest.raises(TypeError):
        rotary.rotate(r, p, q, q.to(BF16))
    with pytest.raises(ValueError):
        rotary.rotate(r, p, q, k_out=q)
    with pytest.raises(ValueError):
        rotary.rotate(r, p, q.transpose(1, 2).contiguous().transpose(1, 2))
    with pytest.raises(binding.PlanError):
        rotary.rotate(r, p, q, out=q[:, :1].expand(5, 2, 64))
