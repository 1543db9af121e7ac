"""The key/value cache in 4 bits on the GPU against its definition in 64 bits (kv4_defs).  Codes,
exponents and values read back have to be the same; attention is held to a bound derived from its
roundings."""
import numpy as np
import pytest
import torch

from gpu_util import host, need_gpu
from kv4_defs import RefCache4, VALUES

pytestmark = pytest.mark.gpu

# half a step of the type, relative to the value (8 and 11 significant bits), and half of its smallest step
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST_STEP = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


class Setup:
    """A cache and its reference, sequences with blocks in any order of the pool."""

    def __init__(self, lengths, *, heads=2, dim=128, block=64, seed=0, spare=2, garbage=True):
        need_gpu()
        from paper_2203_00448_amd import kv
        self.kv = kv
        self.rng = np.random.default_rng([seed, heads, dim, block])
        self.block, self.heads, self.dim = block, heads, dim
        pages = [(n + block - 1) // block for n in lengths]
        n_blocks = max(1, sum(pages) + spare)
        order = self.rng.permutation(n_blocks)
        # entries past a sequence's last token are never read: an index far out says so
        self.table = np.full((len(lengths), max(pages) + 1), 1 << 30, np.int64)
        at = 0
        for s, n in enumerate(pages):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.capacity = list(lengths)
        self.ref = RefCache4(n_blocks, heads, dim, block)
        if garbage:  # never written: the largest codes, scales that are no numbers
            self.ref.k_code[:], self.ref.v_code[:] = 0x7f, 0xf7
            self.ref.k_exp[:], self.ref.v_exp[:] = 255, 255
        c = [torch.from_numpy(getattr(self.ref, x).copy()).cuda() for x in ("k_code", "v_code", "k_exp", "v_exp")]
        self.cache = kv.Cache(*c, kind=kv.E2M1)
        self.d_table = torch.from_numpy(self.table.astype(np.int32)).cuda()

    def seqs(self, length, new=None, **more):
        """(Seqs, begin on the host): `new` rows of each sequence, None for the form of one each."""
        begin = np.concatenate([[0], np.cumsum(np.ones(len(length), np.int64) if new is None else new)])
        b = None if new is None else torch.from_numpy(begin.astype(np.int64)).cuda()
        return self.kv.Seqs(self.d_table, torch.tensor(length, dtype=torch.int32, device="cuda"), begin=b,
                            tokens=int(begin[-1]), **more), begin

    def rows(self, n, heads=None, dtype=BF16, size=1.0):
        x = self.rng.standard_normal((n, heads or self.heads, self.dim)) * size
        x *= 2.0 ** self.rng.integers(-2, 3, (n, heads or self.heads, 1))
        return torch.from_numpy(x).to(dtype).cuda()

    def store(self, length, new, k, v):
        seqs, begin = self.seqs(length, new)
        self.kv.write(self.cache, seqs, k, v)
        self.ref.write(self.table, length, begin, host(k.double()), host(v.double()))

    def write(self, length, new=None, dtype=BF16):
        total = len(length) if new is None else sum(new)
        self.store(length, new, self.rows(total, dtype=dtype), self.rows(total, dtype=dtype))

    def fill(self):
        self.write(self.capacity, self.capacity)

    def same(self):
        """Every byte: what the calls wrote, and what they left."""
        for name in ("k_code", "v_code", "k_exp", "v_exp"):
            assert np.array_equal(host(getattr(self.cache, name)), getattr(self.ref, name)), name

    def attend(self, length, new, q, *, weights, scale=None, lse=True, **more):
        seqs, begin = self.seqs(length, new, **more)
        scale = self.dim ** -0.5 if scale is None else scale
        got = torch.full(q.shape[:2], 7.0, dtype=F32, device="cuda") if lse else None
        out = self.kv.attend(self.cache, seqs, q, scale=scale, lse=got)
        near(out, got, self.ref.attend(self.table, length, begin, host(q.double()), scale), q.dtype, weights)
        return out


# The rounding of a weight: 8 bits; 11 bits; 8 bits and 8 of what these leave.
ONE, HALF, TWO = 2.0 ** -8, 2.0 ** -11, 2.0 ** -15


def most_by_rows(dtype, dim):
    """Rows of a longest piece that go by 16, with weights in two pieces."""
    return 64 if dtype == F16 and dim == 256 else 48


def of_tiles(dtype, dim=128):
    """The rounding where many rows share what is read."""
    return ONE if dtype == BF16 else HALF if dim < 256 else TWO


def near(out, lse, want, dtype, weights):
    """Scores: `dim` products summed in 32 bits and a few roundings more, each 2^-24 of the sum of
    |products| (delta); a weight is off by that times itself, and once more in the sum of weights.
    Weights are rounded (`weights`) and have 2^-20 from the exponential and the sums.  The largest of a row
    is 2^-24 at least, and what is below 2^-126, the least that a float has all its bits at, may be zero: a
    weight, relative to the largest, and its product with a value by 2^-102 each (`floor`: times the sum of 1 + |v|).
    Weights of 11 bits end in steps of 2^-24 where the largest is 2^10 at least: half a step is 2^-35 of it; values
    beside them end in these steps too, half of one 2^-25.  The result is rounded once, in steps that end."""
    ref, ref_lse, mass, delta, floor = want
    score = (ref.shape[-1] + 8) * 2.0 ** -24 * delta[..., None]
    bound = HALF_STEP[dtype] * np.abs(ref) + (weights + 2.0 ** -20 + 2.5 * score) * mass * 1.01 + LEAST_STEP[dtype]
    bound += (2.0 ** -35 if weights == HALF else 2.0 ** -102) * floor + (2.0 ** -25 if weights == HALF else 0.0)
    off = np.abs(host(out.double()) - ref)
    assert np.all(off <= bound), (off / bound).max()
    if lse is not None:
        got, none = host(lse.double()), np.isinf(ref_lse)
        assert np.array_equal(got[none], ref_lse[none])
        room = score[..., 0][~none] + 2.0 ** -20 * (1 + np.abs(ref_lse[~none]))
        assert np.all(np.abs(got[~none] - ref_lse[~none]) <= room)


# ---- write and read


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("block,dim,heads", [(16, 64, 1), (32, 128, 3), (64, 128, 8), (64, 256, 2), (16, 256, 5)])
def test_write_prompts_then_tokens(block, dim, heads, dtype):
    s = Setup([70, 1, 16, 200, 33], heads=heads, dim=dim, block=block)
    s.write([60, 0, 15, 190, 31], [60, 0, 15, 190, 31], dtype)
    s.same()
    s.write([65, 1, 16, 190, 33], [5, 1, 1, 0, 2], dtype)
    s.write([66, 1, 16, 191, 33], None, dtype)  # rewrites the last tokens of three
    s.same()


def test_every_code_and_tie():
    """Every multiple of an eighth up to 7, the group's largest 7 and 6: each code, each halfway case."""
    s = Setup([64], heads=1, dim=64, garbage=False)
    x = np.zeros((64, 1, 64))
    steps = np.arange(64) % 57 / 8.0
    x[:, 0, :] = steps[:, None]
    x[:, 0, 31] = 7.0
    x[:, 0, 63] = -6.0
    x[::2] *= 2.0 ** 100
    x[1::2] *= -2.0 ** -60
    t = torch.from_numpy(x).to(BF16).cuda()
    assert np.array_equal(host(t.double()), x)
    s.store([64], [64], t, t.flip(0).contiguous())
    s.same()


def test_ends_of_the_scale():
    s = Setup([8], heads=1, dim=64, garbage=False)
    x = np.zeros((8, 1, 64))
    x[0, 0, :32], x[0, 0, 32:] = 2.0 ** -126, 3.0e38
    x[1, 0, :32], x[1, 0, 32:] = 7.0 * 2.0 ** 120, 7.03125 * 2.0 ** 120
    x[2, 0, :32], x[2, 0, 32:] = 7.0 * 2.0 ** -100, 0.25 * 2.0 ** -100
    x[3, 0, 0], x[3, 0, 32] = -1.0e-44, 1.0e-38
    x[4, 0, 5], x[5, 0, 63] = 7.0, 7.0000005
    t = torch.from_numpy(x).to(F32).cuda()
    s.store([8], [8], t, -t)
    s.same()


@pytest.mark.parametrize("new", [None, [3]])
def test_write_not_finite(new):
    s = Setup([9], heads=2, garbage=False)
    s.write([6], [6])
    n = 1 if new is None else 3
    k, v = s.rows(n), s.rows(n)
    k[-1, 0, 3], k[-1, 0, 40], v[-1, 1, 7], v[-1, 1, 70] = float("inf"), float("nan"), float("-inf"), float("nan")
    seqs, begin = s.seqs([6 + n], new)
    from paper_2203_00448_amd import binding
    with pytest.raises(binding.PlanError) as e:
        s.kv.write(s.cache, seqs, k, v)
    assert e.value.status == binding.MP_EINVAL
    s.ref.write(s.table, [6 + n], begin, host(k.double()), host(v.double()))
    s.same()


@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 8), (8, 3)])
def test_strided_rows(offset, pad):
    """Rows inside wider ones, aligned and not; heads outside tokens; one row for all tokens."""
    s = Setup([50, 7], heads=3)
    wide = torch.randn(57, 3, 128 + offset + pad, device="cuda").to(BF16)
    k = wide[..., offset:offset + 128]
    v = torch.randn(3, 57, 128, device="cuda").to(BF16).transpose(0, 1)
    s.store([50, 7], [50, 7], k, v)
    s.same()
    seqs, begin = s.seqs([50, 7], [20, 7])
    room = torch.full((27, 3, 128 + offset + pad), 9.0, dtype=F32, device="cuda")
    out = room[..., offset:offset + 128], torch.empty(3, 27, 128, dtype=F32, device="cuda").transpose(0, 1)
    s.kv.read(s.cache, seqs, out=out)
    want = s.ref.read(s.table, [50, 7], begin)
    assert np.array_equal(host(out[0]), want[0]) and np.array_equal(host(out[1]), want[1])
    assert bool((room[..., offset + 128:] == 9).all()) and bool((room[..., :offset] == 9).all())
    same = torch.randn(1, 3, 128, device="cuda").to(F16).expand(57, 3, 128)
    s.store([50, 7], [50, 7], same, same)
    s.same()


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("block,dim", [(16, 64), (32, 256), (64, 128)])
def test_read(block, dim, dtype):
    length = [100, 1, 64, 0, 37]
    s = Setup(length, block=block, dim=dim)
    s.fill()
    for new in (None, [100, 1, 64, 0, 37], [3, 0, 64, 0, 37]):
        if new is None:
            length = [100, 1, 64, 5, 37]  # the form of one token of each: a fourth sequence that has some
            s = Setup(length, block=block, dim=dim)
            s.fill()
        else:
            length = [100, 1, 64, 0, 37]
        seqs, begin = s.seqs(length, new)
        k, v = s.kv.read(s.cache, seqs, dtype=dtype)
        want = s.ref.read(s.table, length, begin)
        for got, x in zip((k, v), want):
            assert torch.equal(got.cpu(), torch.from_numpy(x).to(dtype))


# ---- attention


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("block,dim,heads,group", [(64, 128, 2, 4), (16, 64, 3, 7), (32, 256, 1, 16), (64, 128, 1, 33),
                                                   (16, 128, 5, 1), (64, 64, 2, 8), (16, 256, 2, 3)])
def test_attend_token(block, dim, heads, group, dtype):
    length = [1, 2, 63, 64, 65, 200, 777, 130]
    s = Setup(length, heads=heads, dim=dim, block=block)
    s.fill()
    s.attend(length, None, s.rows(len(length), heads * group, dtype), weights=TWO)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("block,dim,heads,group,new", [
    (64, 128, 2, 4, [300, 1, 64, 17, 100]), (16, 64, 3, 7, [33, 1, 20, 5, 100]), (32, 256, 1, 2, [200, 1, 64, 0, 90]),
    (16, 128, 1, 1, [130, 1, 64, 17, 100]), (64, 64, 2, 3, [300, 1, 64, 17, 100]), (64, 128, 2, 1, [3, 1, 2, 0, 16])])
def test_attend_prompt(block, dim, heads, group, dtype, new):
    length = [300, 1, 64, 257, 100]
    s = Setup(length, heads=heads, dim=dim, block=block)
    s.fill()
    q = s.rows(sum(new), heads * group, dtype)
    # the bounds that the handle gives where none are named: all rows one sequence's, a whole row of the table
    piece, longest = sum(new) * group, s.table.shape[1] * block
    few = piece <= 16 or (piece <= most_by_rows(dtype, dim) and longest > 512)
    s.attend(length, new, q, weights=TWO if few else of_tiles(dtype, dim))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("new", [[9, 1, 2], [10, 1, 2], [1, 0, 15], [12, 2, 3]])
def test_attend_pieces_of_either_form(new, dim, dtype):
    """48, 52, 64 and 68 rows after up to 700 tokens."""
    length = [700, 30, 657]
    s = Setup(length, heads=2, dim=dim)
    s.fill()
    few = sum(new) * 4 <= most_by_rows(dtype, dim)
    s.attend(length, new, s.rows(sum(new), 8, dtype), weights=TWO if few else of_tiles(dtype, dim))


@pytest.mark.parametrize("dtype,dim", [(BF16, 128), (F16, 64), (BF16, 256)])
@pytest.mark.parametrize("group,each", [(4, 1), (4, 2), (4, 4), (4, 3), (7, 3), (7, 2), (16, 3), (8, 5)])
def test_attend_alike(group, each, dim, dtype):
    """As many new tokens of every sequence: row groups in their order."""
    from paper_2203_00448_amd import binding

    length = [700, 30, 657, 64, 5200, 5, 16]
    s = Setup(length, heads=2, dim=dim)
    s.fill()
    n = len(length) * each
    bounds = {"most_new": each, "longest": 5200}
    s.attend(length, [each] * 7, s.rows(n, 2 * group, dtype), weights=TWO, **bounds)
    for new in ([0, 0, 0, 1, 0, 0, 0], [each, each, each, each, each, each, 0], [0] * 7):
        # bounds that end before the rows do: the call says so; no row but theirs is written
        begin = np.concatenate([[0], np.cumsum(new)])
        q = s.rows(n, 2 * group, dtype)
        seqs = s.kv.Seqs(s.d_table, torch.tensor(length, dtype=torch.int32, device="cuda"),
                         begin=torch.from_numpy(begin.astype(np.int64)).cuda(), tokens=n, **bounds)
        out, lse = torch.full_like(q, 3.0), torch.full(q.shape[:2], 7.0, dtype=F32, device="cuda")
        with pytest.raises(binding.PlanError):
            s.kv.attend(s.cache, seqs, q, scale=dim ** -0.5, out=out, lse=lse)
        end = int(begin[-1])
        assert bool((out[end:] == 3.0).all()) and bool((lse[end:] == 7.0).all())


@pytest.mark.parametrize("dtype,dim,length,new", [(BF16, 128, [5000], None), (F16, 64, [9000, 3000], None),
                                                  (BF16, 128, [20000, 100], [40, 40]), (F16, 256, [6000], [3]),
                                                  (BF16, 64, [7000], [100]), (BF16, 128, [9001], [33]),
                                                  (F16, 128, [9001], [40]), (F16, 64, [10000], [65]),
                                                  (F16, 256, [5000, 2000], [30, 70]), (BF16, 256, [8999], [25])])
def test_attend_chunks(dtype, dim, length, new):
    """Long sequences in chunks that are joined; the last chunks of the shorter ones see nothing."""
    s = Setup(length, heads=1, dim=dim)
    s.fill()
    n = len(length) if new is None else sum(new)
    few = new is None or sum(new) * 4 <= most_by_rows(dtype, dim)
    s.attend(length, new, s.rows(n, 4, dtype), weights=TWO if few else of_tiles(dtype, dim))


@pytest.mark.parametrize("block", [16, 64])
@pytest.mark.parametrize("length,new,heads", [
    ([1100] + [1 + i % 70 for i in range(120)], [1100] + [1 + i % 70 for i in range(120)], 8),
    ([1300], [1100], 64), ([5] * 60 + [1500, 40], [9] * 60 + [1030, 60], 17)])
def test_attend_many_prompts(length, new, heads, block):
    """Calls of over a thousand workgroups of 256 rows: teams of waves in turn, sequences in order or by what they
    see, rows that see nothing, tokens of sizes far apart."""
    s = Setup(length, heads=heads, block=block)
    k, v = s.rows(sum(length)), s.rows(sum(length))
    v[::7] *= 2.0 ** 40
    v[:, :, 64:96] *= 2.0 ** -60
    k[::5, :, :32] *= 2.0 ** -20
    s.store(length, length, k, v)
    assert (sum(new) * 4 // 256 + len(new)) * heads >= 1024 and max(new) * 4 >= 4096
    s.attend(length, new, s.rows(sum(new), heads * 4), weights=ONE)


def test_rows_that_see_nothing():
    """More rows than tokens: the first ones see nothing; an empty sequence."""
    s = Setup([5, 70, 40], heads=2)
    s.fill()
    q = s.rows(9 + 90 + 3, 4)
    out = s.attend([5, 70, 0], [9, 90, 3], q, weights=ONE)
    assert bool((out[:4] == 0).all()) and bool((out[9:29] == 0).all()) and bool((out[99:] == 0).all())
    q = s.rows(3, 4)
    out = s.attend([5, 0, 0], None, q, weights=TWO)
    assert bool((out[1:] == 0).all())


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0 ** 40, 2.0 ** -40])
@pytest.mark.parametrize("new", [None, [100]])
def test_scales(scale, new):
    s = Setup([300], heads=1)
    s.fill()
    q = s.rows(1 if new is None else 100, 4)
    if scale == 2.0 ** 40:
        q = (q.float() * 2.0 ** -40).to(BF16)
    s.attend([300], new, q, scale=scale, weights=TWO if new is None else ONE)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("new", [None, [200]])
def test_values_of_sizes_far_apart(new, dtype):
    """Tokens whose values are 2^60 times their neighbours', later than a row or of small weight, cost the row
    nothing; nor do groups of dims of other sizes."""
    s = Setup([200], heads=1)
    k, v = s.rows(200), s.rows(200)
    v[150:153] *= 2.0 ** 60
    v[:, :, 32:64] *= 2.0 ** -50
    k[:, :, 64:96] *= 2.0 ** -30
    s.store([200], [200], k, v)
    q = s.rows(1 if new is None else 200, 4, dtype)
    if dtype == F16:  # the results are no 16-bit floats
        v[150:153] *= 2.0 ** -55
        v[:, :, 32:64] *= 2.0 ** 45
        s.store([200], [200], k, v)
    s.attend([200], new, q, weights=TWO if new is None else of_tiles(dtype))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("odd", [[0], [1], [2, 3], [4], [0, 1, 2, 3, 4]])
def test_scales_that_16_bit_floats_do_not_hold(odd, dim):
    """Rows of 16-bit floats: steps of 64 tokens whose keys or values lie outside that type's range, beside others
    within it; values beyond it with weights that bring them back; groups of zeros, which no scale disturbs."""
    s = Setup([300], heads=1, dim=dim)
    k, v = s.rows(300, size=0.25).float(), s.rows(300).float()
    k[7], v[9] = 0.0, 0.0
    v[130, :, :32] = 0.0
    for t in odd:
        at = slice(64 * t, 64 * t + 60)
        k[at, :, 32:64] *= 2.0 ** -30
        v[at] *= 2.0 ** -27
        v[64 * t + 5] = 400000.0
        k[64 * t + 5] = -1.0
    s.store([300], [300], k.to(BF16), v.to(BF16))
    q = (s.rows(200, 4, F16, size=0.1).float() + 2.0).to(F16)
    # a score of -2 sqrt(dim) and more below the others: at most e^-16 of the weights, with any of these values
    s.attend([300], [200], q, weights=of_tiles(F16, dim))
    s.attend([300], [200], -q, scale=-(dim ** -0.5), weights=of_tiles(F16, dim))
    s.attend([300], None, q[:1], weights=TWO)


@pytest.mark.parametrize("new", [None, [70]])
def test_large_and_small_queries_and_keys(new):
    s = Setup([130], heads=2)
    k, v = s.rows(130), s.rows(130)
    k[:, 0] *= 2.0 ** 100
    k[:, 1] *= 2.0 ** -90
    s.store([130], [130], k, v)
    q = s.rows(2 if new is None else 70, 4)[:1 if new is None else 70]
    q[:, :2] *= 2.0 ** -98
    q[:, 2:] *= 2.0 ** 92
    s.attend([130], new, q, weights=TWO if new is None else ONE)


@pytest.mark.parametrize("new", [None, [90]])
def test_scores_of_thousands(new):
    """One key far above the others; scores beyond 2^16 whose differences are small."""
    s = Setup([256], heads=1)
    k, v = s.rows(256), s.rows(256)
    k[100] *= 64.0
    s.store([256], [256], k, v)
    q = s.rows(1 if new is None else 90, 4) * 16
    out = s.attend([256], new, q, weights=TWO if new is None else ONE)
    assert bool(torch.isfinite(out).all())
    k[:] = 1.0
    k[:, :, 0] = 0.5 + torch.arange(256, device="cuda").view(-1, 1) % 2
    s.store([256], [256], k, v)
    q[:] = 0.0
    q[:, :, 1], q[:, :, 0] = 2.0 ** 17, 1.0
    seqs, begin = s.seqs([256], new)
    out = s.kv.attend(s.cache, seqs, q, scale=1.0)
    # scores 2^17 + 0.5 or + 1.5: whole multiples of 2^-1, exact in 32 bits; times log2 e they are off by
    # 2^-7 (half of the last place of 2^17.6), and the scale's own rounding is the same for all but for a difference
    # of one times 2^-24: a weight is off by ln 2 times 2^-7
    ref, _, mass, _, _ = s.ref.attend(s.table, [256], begin, host(q.double()), 1.0)
    bound = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2 * 0.7 * 2.0 ** -7) * mass * 1.02
    assert np.all(np.abs(host(out.double()) - ref) <= bound)


@pytest.mark.parametrize("dtype,new", [(BF16, None), (F16, [150]), (BF16, [150])])
def test_repeats_and_views(dtype, new):
    """The same bits again, on another stream, into strided views, with a workspace and without the logarithms."""
    s = Setup([700, 150], heads=2)
    s.fill()
    new = None if new is None else [40, 150]
    n = 2 if new is None else sum(new)
    wide = torch.randn(n, 2, 8, 136, device="cuda").to(dtype)
    q = wide[:, 1, :, :128]
    want = s.attend([700, 150], new, q, weights=TWO if new is None else of_tiles(dtype))
    seqs, _ = s.seqs([700, 150], new)
    room = torch.full((n, 9, 130), 5.0, dtype=dtype, device="cuda")
    out = room[:, :8, 1:129]
    ws = s.kv.workspace(s.kv.OP_ATTEND, s.cache, seqs, q_heads=8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = s.kv.attend(s.cache, seqs, q, out=out, workspace=ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert got is out and torch.equal(out, want)
    assert bool((room[:, 8] == 5).all()) and bool((room[..., 0] == 5).all()) and bool((room[..., 129:] == 5).all())


@pytest.mark.parametrize("dtype,length,new", [(BF16, [3000, 900], None), (F16, [5000, 64], [100, 30]),
                                              (BF16, [4000, 700], [60, 700])])
def test_recorded(dtype, length, new):
    """A write and an attention in chunks in one graph, replayed with other rows, eager work between."""
    a, b = Setup(length, heads=2), Setup(length, heads=2)
    a.fill()
    for x, y in zip(a.cache.tensors, b.cache.tensors):
        y.copy_(x)
    n = 2 if new is None else sum(new)
    seqs = [s.seqs(length, new)[0] for s in (a, b)]
    q, k, v = a.rows(n, 8, dtype), a.rows(n, 2, dtype), a.rows(n, 2, dtype)
    ws = [s.kv.workspace(s.kv.OP_ATTEND, s.cache, x, q_heads=8) for s, x in zip((a, b), seqs)]
    status, outs = a.kv.new_status(), [torch.zeros_like(q) for _ in range(2)]

    def both(s, x, space, out):
        s.kv.write(s.cache, x, k, v, status=status, check=False)
        s.kv.attend(s.cache, x, q, out=out, workspace=space, status=status, check=False)

    both(a, seqs[0], ws[0], outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(a, seqs[0], ws[0], outs[0])
    for i in range(5):
        for t, rows in ((q, a.rows(n, 8, dtype)), (k, a.rows(n, 2, dtype)), (v, a.rows(n, 2, dtype))):
            t.copy_(rows)
        graph.replay()
        both(b, seqs[1], ws[1], outs[1])
        assert torch.equal(outs[0], outs[1]), i
        assert all(torch.equal(x, y) for x, y in zip(a.cache.tensors, b.cache.tensors))
    assert int(status.item()) == 0


def test_places_past_32_bits():
    """Blocks whose codes lie more than 2^32 bytes into a cache, table rows and query rows as far apart."""
    need_gpu()
    from paper_2203_00448_amd import kv
    n_blocks, dim = (1 << 20) + 5, 128
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("not enough memory")
    c = [torch.empty(n_blocks, 1, 64, dim // 2, dtype=torch.uint8, device="cuda") for _ in range(2)]
    c += [torch.empty(n_blocks, 1, dim // 32, 64, dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = kv.Cache(*c, kind=kv.E2M1)
    wide = torch.zeros(2, (1 << 30) + 3, dtype=torch.int32, device="cuda")
    table = wide[:, :3]
    table[0] = torch.tensor([n_blocks - 1, 3, n_blocks - 2])
    table[1] = torch.tensor([n_blocks - 4, n_blocks - 3, 0])
    s = Setup([150, 100], heads=1, garbage=False)
    for x, y in zip(s.table, ([n_blocks - 1, 3, n_blocks - 2], [n_blocks - 4, n_blocks - 3])):
        s.order = getattr(s, "order", {}) | {int(b): int(f) for b, f in zip(x, y)}
    rows = torch.zeros(2 * (1 << 31) + 4096, dtype=BF16, device="cuda")
    q = rows.as_strided((250, 1, 128), (1 << 24, 128, 1))
    q.copy_(s.rows(250))
    k, v = s.rows(250), s.rows(250)
    length = torch.tensor([150, 100], dtype=torch.int32, device="cuda")
    begin = torch.tensor([0, 150, 250], dtype=torch.int64, device="cuda")
    seqs = kv.Seqs(table, length, begin=begin, tokens=250)
    kv.write(cache, seqs, k, v)
    s.ref.write(s.table, [150, 100], [0, 150, 250], host(k.double()), host(v.double()))
    for small, far in s.order.items():
        if far != 0:
            got = host(cache.k_code[far])
            used = 64 if far not in (n_blocks - 2, n_blocks - 3) else (150 - 128 if far == n_blocks - 2 else 100 - 64)
            assert np.array_equal(got[:, :used], s.ref.k_code[small][:, :used])
    near(kv.attend(cache, seqs, q), None, s.ref.attend(s.table, [150, 100], [0, 150, 250], host(q.double()), dim ** -0.5),
         BF16, ONE)
    ones = kv.Seqs(table, length)
    got = kv.attend(cache, ones, q[:2])
    near(got, None, s.ref.attend(s.table, [150, 100], [0, 1, 2], host(q[:2].double()), dim ** -0.5), BF16, TWO)
    back = kv.read(cache, seqs, dtype=F32)
    want = s.ref.read(s.table, [150, 100], [0, 150, 250])
    assert np.array_equal(host(back[0]), want[0]) and np.array_equal(host(back[1]), want[1])


def test_rows_behind_the_last_sequence_are_left():
    """A padded batch: sequences of no rows at the end, rows that are no sequence's."""
    s = Setup([90, 20, 30], heads=1)
    s.fill()
    begin = torch.tensor([0, 40, 40, 40], dtype=torch.int64, device="cuda")
    seqs = s.kv.Seqs(s.d_table, torch.tensor([90, 20, 30], dtype=torch.int32, device="cuda"), begin=begin, tokens=40)
    q = s.rows(60, 4)
    out = torch.full_like(q, 3.0)
    s.kv.attend(s.cache, seqs, q[:40], out=out[:40])
    assert bool((out[40:] == 3).all())
    near(out[:40], None, s.ref.attend(s.table, [90, 20, 30], [0, 40, 40, 40], host(q[:40].double()), 128 ** -0.5),
         BF16, ONE)


def test_bad_pages_and_bounds():
    """Table entries and bounds outside their ranges raise the status word."""
    s = Setup([100, 40], heads=1)
    s.fill()
    from paper_2203_00448_amd import binding
    bad = s.d_table.clone()
    for entry in (-1, s.cache.n_blocks, 1 << 30):
        bad[1, 0] = entry
        for new in (None, [20, 20]):
            begin = None if new is None else torch.tensor([0, 20, 40], dtype=torch.int64, device="cuda")
            seqs = s.kv.Seqs(bad, torch.tensor([100, 40], dtype=torch.int32, device="cuda"), begin=begin)
            n = 2 if new is None else 40
            rows = torch.zeros(n, 1, 128, dtype=BF16, device="cuda")
            for call in (lambda: s.kv.attend(s.cache, seqs, rows), lambda: s.kv.read(s.cache, seqs)):
                with pytest.raises(binding.PlanError) as e:
                    call()
                assert e.value.status == binding.MP_EINVAL
    seqs = s.kv.Seqs(s.d_table, torch.tensor([5, 40], dtype=torch.int32, device="cuda"),
                     begin=torch.tensor([0, 10, 20], dtype=torch.int64, device="cuda"))
    with pytest.raises(binding.PlanError):  # more rows than tokens
        s.kv.write(s.cache, seqs, *(torch.zeros(20, 1, 128, dtype=BF16, device="cuda") for _ in range(2)))
    s.ref.write(s.table, [5, 40], [0, 0, 10], np.zeros((10, 1, 128)), np.zeros((10, 1, 128)))
    s.same()


def test_refusals():
    need_gpu()
    from paper_2203_00448_amd import binding, kv
    c = kv.new_cache(4, 2, 128, kind=kv.E2M1)
    assert c.nbytes == 2 * 4 * 2 * 64 * (64 + 4)
    seqs = kv.Seqs(torch.zeros(1, 4, dtype=torch.int32, device="cuda"),
                   torch.ones(1, dtype=torch.int32, device="cuda"))
    q = torch.zeros(1, 4, 128, dtype=BF16, device="cuda")
    with pytest.raises(binding.PlanError):
        kv.select(c, seqs, q, keep=2)
    with pytest.raises(binding.PlanError):
        kv.attend(c, seqs, q, blocks=torch.zeros(1, 2, 1, dtype=torch.int32, device="cuda"))
    with pytest.raises(TypeError):
        kv.attend(c, seqs, q.float())
    with pytest.raises(ValueError):
        kv.Cache(*c.tensors, c.k_exp, kind=kv.E2M1)
    with pytest.raises(TypeError):
        kv.Cache(c.k_code, c.v_code, c.k_exp.view(torch.int8), c.v_exp, kind=kv.E2M1)
    with pytest.raises(ValueError):
        kv.Cache(c.k_code, c.v_code, c.k_exp[:, :, :2].contiguous(), c.v_exp, kind=kv.E2M1)
    with pytest.raises(binding.PlanError):
        kv.write(kv.new_cache(4, 2, 96, kind=kv.E2M1), seqs, *(torch.zeros(1, 2, 96, dtype=BF16, device="cuda"),) * 2)


def test_the_reference_itself():
    from kv4_defs import encode4, least_exponent4
    assert [int(x) for x in encode4(VALUES)] == list(range(16))
    assert list(encode4(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25]))) == [0, 2, 2, 4, 4, 6, 6, 7, 8]
    for top in (1e-3, 0.5, 6.0, 7.0, 7.01, 448.0, 1e30):
        e = least_exponent4(top)
        assert top <= 7.0 * 2.0 ** e and top > 7.0 * 2.0 ** (e - 1)
