"""The ends of the ranges that the 4-bit cache's attention takes: values, keys, queries and scales whose products or
sums in 32 bits could leave the range of such floats although the result does not, in each form of the kernel."""
import numpy as np
import pytest
import torch

from gpu_util import host
from test_gpu_kv4 import BF16, F16, HALF, HALF_STEP, LEAST_STEP, ONE, TWO, Setup, of_tiles

pytestmark = pytest.mark.gpu


def attend(s, length, new, q, scale):
    seqs, begin = s.seqs(length, new)
    out = s.kv.attend(s.cache, seqs, q, scale=scale)
    return host(out.double()), s.ref.attend(s.table, length, begin, host(q.double()), scale)


def within(out, want, dtype, weights, dims=slice(None), more=0.0):
    """The bound of test_gpu_kv4.near for some of the dims, and `more`."""
    ref, _, mass, delta, floor = want
    score = (ref.shape[-1] + 8) * 2.0 ** -24 * delta[..., None]
    ref, mass, floor = ref[..., dims], mass[..., dims], floor[..., dims]
    bound = HALF_STEP[dtype] * np.abs(ref) + (weights + 2.0 ** -20 + 2.5 * score) * mass * 1.01 + LEAST_STEP[dtype]
    bound += (2.0 ** -35 if weights == HALF else 2.0 ** -102) * floor + (2.0 ** -25 if weights == HALF else 0.0) + more
    off = np.abs(out[..., dims] - ref)
    assert np.all(off <= bound), (off / bound).max()  # also where it is no number


def filled(dim, far, size, key, largest):
    """300 tokens of a head; the key of token 70 far above the others'; one token of each of the steps `far` with values
    of `size` in dims 32 to 63 and with the keys `key`."""
    s = Setup([300], heads=1, dim=dim)
    k, v = s.rows(300, size=0.25).float(), s.rows(300).float()
    tokens = [64 * t + 3 for t in far]
    k[70] = largest
    for t in tokens:
        k[t] = key
        v[t, :, 32:64] = size
    s.store([300], [300], k.to(BF16), v.to(BF16))
    return s, tokens


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("size", [2.0 ** 120, -6.0 * 2.0 ** 120, 2.0 ** 100])
@pytest.mark.parametrize("far", [[0], [1], [2], [4], [0, 2], [0, 1, 2, 3, 4]])
def test_large_values_that_others_outweigh(far, size, dim):
    """Rows of 16-bit floats over values that these do not hold, the most weight of their steps (keys of 1) and none
    beside a key of 16 that comes later or came before: exp(-15 * 2 sqrt(dim)) < 2^-340 of the sum, below 2^-200
    with any of these values.  So the result is that without them, to 2^-60."""
    s, tokens = filled(dim, far, size, 1.0, 16.0)
    q = (s.rows(200, 4, F16, size=0.01).float() + 2.0).to(F16)
    length, begin = [300], [0, 200]
    for t in tokens:  # the definition without them
        s.ref.v_code[s.table[0][t // 64], :, t % 64] = 0
    for sign in (1.0, -1.0):
        out, want = attend(s, length, [200], sign * q, sign * dim ** -0.5)
        within(out, want, F16, of_tiles(F16, dim), more=2.0 ** -60)
    out, want = attend(s, length, None, q[-1:], dim ** -0.5)
    within(out, want, F16, TWO, more=2.0 ** -60)


@pytest.mark.parametrize("dim,key,size", [(64, [4.0, 4.0], 2.0 ** 100), (128, [6.0, 4.0], 2.0 ** 104),
                                          (256, [6.0, 6.0], 2.0 ** 100)])
@pytest.mark.parametrize("far", [[0], [2], [1, 3]])
def test_large_values_of_small_weight(far, dim, key, size):
    """Shares of 2^-90 to 2^-98 that the values bring back into range, in the steps that hold them and in those
    after."""
    s, _ = filled(dim, far, size, torch.tensor(key, device="cuda").repeat(dim // 2), 8.0)
    q = (2.0 + 2.0 ** -8 * torch.randint(-1, 2, (200, 4, dim), device="cuda").float()).to(F16)
    out, want = attend(s, [300], [200], q, dim ** -0.5)
    assert 1.0 < np.abs(want[0][-1, :, 32:64]).max() < 60000.0
    # weights of 8 and 8 bits bring these dims' mass; what is beside them is less than 2^-4 of it at 11 bits
    within(out, want, F16, TWO, slice(32, 64))
    within(out, want, F16, of_tiles(F16, dim), slice(0, 32))
    if dim > 64:
        within(out, want, F16, of_tiles(F16, dim), slice(64, None))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("new", [None, [130]])
def test_large_queries_and_keys_of_a_tiny_scale(new, dim, dtype):
    """Products of queries and keys past 2^128, which the scale brings back to some units; and a head whose scores all
    but vanish.  (All keys' scales are past what 16-bit floats hold, so their rows' weights have 16 bits in tiles.)"""
    s = Setup([200], heads=2, dim=dim)
    k, v = s.rows(200).float(), s.rows(200)
    k[:, 0] *= 2.0 ** 116
    k[:, 1] *= 2.0 ** -90
    s.store([200], [200], k.to(BF16), v)
    q = s.rows(1 if new is None else 130, 8, dtype, size=2.0 ** 9)
    for scale in (2.0 ** -126, -(2.0 ** -126)):
        out, want = attend(s, [200], new, q, scale)
        within(out, want, dtype, TWO if new is None or dtype == F16 else ONE)


@pytest.mark.parametrize("scale", [0.0, 2.0 ** -149, -(2.0 ** -149), 2.0 ** -137, 2.0 ** -128, 2.0 ** -126])
@pytest.mark.parametrize("dtype,dim,new,heads", [
    (t, d, n, 1) for t in (BF16, F16) for d in (64, 128, 256) for n in (None, 130)] + [(BF16, 128, 1030, 60)])
def test_the_largest_keys_beside_no_scale(dtype, dim, new, heads, scale):
    """Keys of the largest size, of either sign, whose products with the queries are near 2^128: a scale of zero makes
    their scores zero, and the least ones less than 2^-10.  (1030 rows of 60 heads: teams of waves in turn.)"""
    n = new or 200
    s = Setup([n], heads=heads, dim=dim)
    k, v = s.rows(n).float(), s.rows(n)
    k[:] = 6.0 * 2.0 ** 120
    k[::3] *= -1.0
    s.store([n], [n], k.to(BF16), v)
    rows = 1 if new is None else n
    q = (2.0 + 2.0 ** -4 * torch.randint(-8, 9, (rows, 4 * heads, dim), device="cuda").float()).to(dtype)
    out, want = attend(s, [n], None if new is None else [n], q, scale)
    within(out, want, dtype, TWO if new is None or dtype == F16 else ONE)


LENGTHS = [(t, d, 300, n, 4, 1) for t in (BF16, F16) for d in (64, 128, 256) for n in (None, 130)]
LONG = [(BF16, 128, 5000, None, 4, 1), (F16, 64, 9000, 65, 4, 1), (BF16, 256, 6000, 40, 4, 1), (F16, 128, 7000, 9, 2, 2)]


@pytest.mark.parametrize("dtype,dim,length,new,group,heads,power", [
    (*x, p) for p in (10, 15, 17, 20, 24, 26, 27, 28, 29, 30, 31, 33, 48, 90, 115) for x in LENGTHS] + [
    (*x, p) for p in (20, 28, 31, 90) for x in LONG] + [(BF16, 128, 1030, 1030, 4, 60, p) for p in (20, 31)])
def test_scores_of_any_size(dtype, dim, length, new, group, heads, power):
    """Scores up to 2^(power + 1) beside ones of about one, in the same steps and in others, and a few tokens whose scores are
    the same largest one: those share all the weight, whatever their last places are rounded to.

    The largest keys are all ones (exact: codes of 1); the others of that size have two dims or more of another value,
    so their scores are 2^(power - 8) lower at least (dim is 256 at most), where the arithmetic of a score is off by
    (dim + 8) 2^-24 of it: less than a sixteenth of that.  Equal keys have the same error."""
    s = Setup([length], heads=heads, dim=dim)
    rng = np.random.default_rng(power)
    ones = np.ones((length, heads, dim))
    ones[:, :, 3] = ones[:, :, dim - 2] = 0.5
    most = np.flatnonzero(rng.random(length) < 0.03)
    first = length - (new or 1)
    most = np.concatenate([most, [first // 2]])  # every row sees one
    ones[most] = 1.0
    small = rng.random(length) < 0.3
    if length > 4000:  # chunks without a large score
        most = most[most > length // 3]
        small[:length // 3] = True
    small[most] = False
    small[:64] = True
    k = np.where(small[:, None, None], ones * 2.0 ** -power * rng.choice([1.0, -1.0], (length, 1, 1)), ones)
    if first // 2 < 64:
        k[first // 2] = 1.0
    v = s.rows(length)
    s.store([length], [length], torch.from_numpy(k).to(BF16).cuda(), v)
    q = torch.ones(new or 1, heads * group, dim, device="cuda").to(dtype)
    scale = float(np.float32((1.0 + rng.random()) * 2.0 ** power / dim))
    for sign in (1.0, -1.0):
        seqs, begin = s.seqs([length], None if new is None else [new])
        lse = torch.zeros(q.shape[:2], device="cuda")
        out = host(s.kv.attend(s.cache, seqs, sign * q, scale=sign * scale, lse=lse).double())
        ref, ref_lse, mass, _, _ = s.ref.attend(s.table, [length], begin, host(sign * q.double()), sign * scale)
        piece, longest = q.shape[0] * group, s.table.shape[1] * s.block
        few = piece <= 16 or (piece <= (64 if dtype == F16 and dim == 256 else 48) and longest > 512)
        weights = TWO if new is None or few else of_tiles(dtype, dim)
        # a score's own error where the next ones still have weight: below 2^15 (e^-64 and 2^-92 of the rest from there)
        score = 2.5 * (dim + 8) * 2.0 ** -24 * (2.0 ** (power + 1) if power < 14 else 0.0)
        bound = HALF_STEP[dtype] * np.abs(ref) + (weights + 2.0 ** -19 + score) * mass * 1.01 + 2.0 ** -25
        off = np.abs(out - ref)
        assert np.all(off <= bound), (off / bound).max()
        got = host(lse.double())
        room = (dim + 8) * 2.0 ** -24 * 2.0 ** (power + 1) + 2.0 ** -20 * (1 + np.abs(ref_lse))
        assert np.all(np.abs(got - ref_lse) <= room)


@pytest.mark.parametrize("power", [10, 20, 28, 29, 31, 60])
@pytest.mark.parametrize("dim,new", [(64, None), (128, None), (256, None), (64, 130), (128, 130), (256, 130)])
def test_large_values_of_large_scores(dim, new, power):
    """Two hundred tokens of the same score with values near the end of the range: their sum is past it."""
    s = Setup([300], heads=1, dim=dim)
    k, v = torch.ones(300, 1, dim, device="cuda"), torch.full((300, 1, dim), 6.0 * 2.0 ** 120, device="cuda")
    k[::3, :, 5] = 0.5
    v[::3] = -1.0
    s.store([300], [300], k.to(BF16), v.to(BF16))
    q = torch.ones(new or 1, 4, dim, device="cuda").to(BF16)
    out, want = attend(s, [300], None if new is None else [new], q, 2.0 ** power / dim)
    ref = want[0]
    # the others have e^-(2^power / (2 dim)) of the weight, less than 2^-2; a score is off by (dim + 8) 2^-24 of it
    weights = (TWO if new is None else ONE) + 2.0 ** -19 + 2.5 * (dim + 8) * 2.0 ** -14 * (power == 10)
    assert np.all(np.abs(out - ref) <= (2.0 ** -8 + weights * 1.01) * np.abs(want[2]))


@pytest.mark.parametrize("power", [8, 14, 20, 28, 31, 90])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("far", [[0], [2], [0, 2, 4]])
def test_large_values_that_large_scores_outweigh(far, dim, power):
    """Both at once, rows of 16-bit floats: token 70, whose key is 16 where the others' are one or less, has all the
    weight, so the result is its values; rows from 100 on."""
    s, _ = filled(dim, far, 6.0 * 2.0 ** 120, 1.0, 16.0)
    q = torch.full((200, 4, dim), 2.0, dtype=F16, device="cuda")
    q[::7] = 1.0
    v = s.ref.values([s.table[0][1]], 0)[1][70 - 64]
    for sign in (1.0, -1.0):
        seqs, _ = s.seqs([300], [200])
        out = host(s.kv.attend(s.cache, seqs, sign * q, scale=sign * 2.0 ** power / dim).double())
        # the other scores are 15 * 2^power lower or more: e^-3840; what is left is the roundings of a weight and the result
        assert np.all(np.abs(out - v) <= (2.0 ** -11 + of_tiles(F16, dim) + 2.0 ** -19) * np.abs(v))


@pytest.mark.parametrize("dtype,dim,length,new,heads", [
    (t, d, 300, n, 1) for t in (BF16, F16) for d in (64, 128, 256) for n in (None, 10, 200)] + [(BF16, 128, 1100, 1030, 60)])
def test_queries_that_are_no_numbers(dtype, dim, length, new, heads):
    """Infinities and NaN in some queries make those rows NaN and cost the others nothing."""
    s = Setup([length], heads=heads, dim=dim)
    s.fill()
    n = new or 1
    q = s.rows(n, 4 * heads, dtype)
    odd = [(0, 1), (3, 2), (n - 1, 0), (n // 2, 3)] if n > 1 else [(0, 1)]
    bad = q.clone()
    for i, (token, head) in enumerate(odd):
        bad[token, head, i] = (float("nan"), float("inf"), float("-inf"), float("nan"))[i]
    seqs, begin = s.seqs([length], None if new is None else [new])
    got = host(s.kv.attend(s.cache, seqs, bad).double())
    want = s.ref.attend(s.table, [length], begin, host(q.double()), dim ** -0.5)
    for token, head in odd:
        assert np.isnan(got[token, head]).all()
        got[token, head] = want[0][token, head]
    within(got, want, dtype, TWO if new is None else of_tiles(dtype, dim))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("new", [None, 130])
def test_the_smallest_16_bit_queries(new, dim):
    """Multiples of the least such float, and rows of zeros."""
    s = Setup([300], heads=1, dim=dim)
    s.fill()
    n = new or 1
    q = torch.randint(-9, 10, (n, 4, dim), device="cuda").float()
    q[:, 1] *= 100.0
    q[0, 0] = 0.0
    q = (q * 2.0 ** -24).to(F16)
    out, want = attend(s, [300], None if new is None else [new], q, 2.0 ** 17)
    within(out, want, F16, TWO if new is None else of_tiles(F16, dim))
