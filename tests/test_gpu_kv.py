"""The 8-bit key/value cache on the GPU against its definition in 64 bits
(kv_defs.RefCache).  Codes, exponents, means, values read back and selected
blocks have to be the same; attention is held to a bound derived from its
roundings."""
import numpy as np
import pytest
import torch

from gpu_util import host, need_gpu
from kv_defs import E4M3, INT8, RefCache

pytestmark = pytest.mark.gpu

KINDS = [pytest.param(E4M3, id="e4m3"), pytest.param(INT8, id="int8")]
# half a step of the type, relative to the value (8 and 11 significant bits)
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# half of the type's smallest step
LEAST_STEP = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def module():
    need_gpu()
    from paper_2203_00448_amd import kv
    return kv


class Setup:
    """A cache and its reference, sequences with blocks in any order of the pool."""

    def __init__(self, lengths, *, heads=2, dim=128, block=64, kind=E4M3, seed=0, spare=2, garbage=True):
        self.kv = module()
        self.rng = np.random.default_rng([seed, heads, dim, block, kind])
        self.block, self.heads, self.dim, self.kind = block, heads, dim, kind
        pages = [(n + block - 1) // block for n in lengths]
        n_blocks = max(1, sum(pages) + spare)
        order = self.rng.permutation(n_blocks)
        width = max(pages) + 1
        # entries past a sequence's last token are never read: an index far out says so
        self.table = np.full((len(lengths), width), 1 << 30, np.int64)
        at = 0
        for s, n in enumerate(pages):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.capacity = np.array(lengths)
        self.ref = RefCache(n_blocks, heads, dim, block, kind)
        if garbage:  # never written: codes that are NaN, exponents that would show
            self.ref.k_code[:], self.ref.v_code[:] = 0x7f, 0x7f
            self.ref.k_exp[:], self.ref.v_exp[:] = 90, 90
            self.ref.mean_exp[:] = 90
        c = {x: torch.from_numpy(getattr(self.ref, x).copy()).cuda()
             for x in ("k_code", "v_code", "k_exp", "v_exp", "mean_code", "mean_exp")}
        self.cache = self.kv.Cache(*c.values(), kind=kind)
        self.d_table = torch.from_numpy(self.table.astype(np.int32)).cuda()

    def seqs(self, length, new=None, **more):
        """(Seqs, begin on the host): `new` rows of each sequence, None for the form of one each."""
        begin = np.concatenate([[0], np.cumsum(np.ones(len(length), np.int64) if new is None else new)])
        b = None if new is None else torch.from_numpy(begin.astype(np.int64)).cuda()
        return self.kv.Seqs(self.d_table, torch.tensor(length, dtype=torch.int32, device="cuda"), begin=b,
                            tokens=int(begin[-1]), **more), begin

    def rows(self, n, heads=None, dtype=torch.bfloat16, size=1.0):
        heads = heads or self.heads
        x = self.rng.standard_normal((n, heads, self.dim)) * size
        x *= 2.0 ** self.rng.integers(-2, 3, (n, heads, 1))
        return torch.from_numpy(x).to(dtype).cuda()

    def write(self, length, new=None, dtype=torch.bfloat16, size=1.0):
        seqs, begin = self.seqs(length, new)
        k, v = self.rows(int(begin[-1]), dtype=dtype, size=size), self.rows(int(begin[-1]), dtype=dtype, size=size)
        self.kv.write(self.cache, seqs, k, v)
        self.ref.write(self.table, length, begin, host(k.double()), host(v.double()))

    def fill(self, size=1.0):
        """Every sequence to its full length."""
        self.write(list(self.capacity), list(self.capacity), size=size)

    def same(self):
        """All that lies below the sequences' lengths, and the exponents and means."""
        for name in ("k_exp", "v_exp", "mean_code", "mean_exp"):
            assert np.array_equal(host(getattr(self.cache, name)), getattr(self.ref, name)), name

    def same_codes(self, length):
        k, v = host(self.cache.k_code), host(self.cache.v_code)
        for s, n in enumerate(length):
            for b in range((n + self.block - 1) // self.block):
                p, m = self.table[s, b], min(self.block, n - b * self.block)
                assert np.array_equal(k[p, :, :m], self.ref.k_code[p, :, :m]), (s, b)
                assert np.array_equal(v[p, :, :, :m], self.ref.v_code[p, :, :, :m]), (s, b)


def near(out, lse, want, dtype):
    """out against (out, lse, mass, delta) of the reference.

    Scores: `dim` products summed in 32 bits and a few roundings more, each 2^-24 of the sum of
    |products| (delta); a weight is off by that times itself, and once more in the sum of weights.
    Weights are rounded to 11 bits (half a step: 2^-11) and have 2^-22 from the exponential and
    the sums; as 16-bit floats that reach 2^15 they end in steps of 2^-24, so each is also off by
    2^-40 of the largest (`floor`: that times the sum of a dim's largest values).  The result is
    rounded once, in steps that end too."""
    ref, ref_lse, mass, delta, floor = want
    dim = ref.shape[-1]
    score = (dim + 8) * 2.0 ** -24 * delta[..., None]
    bound = HALF_STEP[dtype] * np.abs(ref) + (2.0 ** -11 + 2.0 ** -20 + 2.5 * score) * mass * 1.01
    bound += 2.0 ** -40 * floor[..., None] + LEAST_STEP[dtype]
    off = np.abs(host(out.double()) - ref)
    assert np.all(off <= bound), (off / bound).max()
    if lse is not None:
        got = host(lse.double())
        none = np.isinf(ref_lse)
        assert np.array_equal(got[none], ref_lse[none])
        ok = ~none
        room = score[..., 0][ok] + 2.0 ** -20 * (1 + np.abs(ref_lse[ok]))
        assert np.all(np.abs(got[ok] - ref_lse[ok]) <= room)


# ---- write and read

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("block,dim,heads", [(16, 64, 3), (32, 128, 2), (64, 128, 1), (64, 256, 2), (16, 256, 1)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_write_prompts_then_tokens(kind, block, dim, heads, dtype):
    """Prompts of every length around a block's, then tokens one by one across blocks, of sizes
    that make held scales grow."""
    start = [0, 1, block - 1, block, block + 1, 3 * block, 2 * block + 7]
    s = Setup([n + block + 5 for n in start], heads=heads, dim=dim, block=block, kind=kind)
    s.write(start, start, dtype=dtype)
    s.same()
    s.same_codes(start)
    length = start
    for step in range(block + 5):
        length = [n + 1 for n in length]
        s.write(length, None, dtype=dtype, size=2.0 ** (step % 7 - 3))
    s.same()
    s.same_codes(length)


@pytest.mark.parametrize("kind", KINDS)
def test_write_pieces(kind):
    """Ragged pieces, empty ones among them, that start and end anywhere in a block."""
    s = Setup([500, 3, 200, 64, 129], kind=kind, block=32)
    length = [0] * 5
    for new in ([5, 1, 0, 64, 100], [27, 0, 1, 0, 28], [1, 2, 150, 0, 1], [400, 0, 0, 0, 0], [67, 0, 49, 0, 0]):
        length = [a + b for a, b in zip(length, new)]
        s.write(length, new, size=1.0 + sum(length) % 9)
        s.same()
        s.same_codes(length)


def test_write_zeros_and_extremes():
    """A block of zeros, values of the type's ends, subnormal ones."""
    for kind in (E4M3, INT8):
        s = Setup([64, 64, 64, 64], block=64, kind=kind)
        n = 256
        k = torch.zeros(n, 2, 128)
        k[64:128] = 3.0e38
        k[128:192] = -1e-39
        k[192:256, :, ::2] = 448.0
        k[192:256, :, 1::2] = 2.0 ** -9
        v = -k
        seqs, begin = s.seqs([64] * 4, [64] * 4)
        s.kv.write(s.cache, seqs, k.cuda(), v.cuda())
        s.ref.write(s.table, [64] * 4, begin, k.double().numpy(), v.double().numpy())
        s.same()
        s.same_codes([64] * 4)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new", [None, [40]])
def test_write_not_finite(kind, new):
    """Raised as a data error; held as the largest value and as zero."""
    s = Setup([40], block=32, kind=kind, garbage=False)
    length = [40] if new else [1]
    seqs, begin = s.seqs(length, new)
    k, v = s.rows(int(begin[-1])), s.rows(int(begin[-1]))
    k[0, 0, 3], k[0, 1, 4], v[0, 1, 77] = float("inf"), float("nan"), float("-inf")
    status = s.kv.new_status()
    s.kv.write(s.cache, seqs, k, v, status=status, check=False)
    assert status.item() == -1
    s.ref.write(s.table, length, begin, host(k.double()), host(v.double()))
    s.same()
    s.same_codes(length)


@pytest.mark.parametrize("layout", ["fused", "odd", "heads_first"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_strides(layout, dtype):
    """Rows inside a wider tensor, rows at odd addresses, heads before tokens: in and out."""
    s = Setup([70, 31], block=32, dim=64, heads=3)
    n = 101

    def room():
        if layout == "fused":
            return torch.zeros(n, 3 * 3, 64, dtype=dtype, device="cuda")[:, 3:6]
        if layout == "odd":
            return torch.zeros(n * 3 * 65 + 1, dtype=dtype, device="cuda")[1:].view(n, 3, 65)[..., :64]
        return torch.zeros(3, n, 64, dtype=dtype, device="cuda").transpose(0, 1)

    k, v = room(), room()
    k.copy_(s.rows(n, dtype=dtype))
    v.copy_(s.rows(n, dtype=dtype))
    seqs, begin = s.seqs([70, 31], [70, 31])
    s.kv.write(s.cache, seqs, k, v)
    s.ref.write(s.table, [70, 31], begin, host(k.double()), host(v.double()))
    s.same()
    s.same_codes([70, 31])
    out = room(), room()
    s.kv.read(s.cache, seqs, out=out)
    for got, want in zip(out, s.ref.read(s.table, [70, 31], begin)):
        assert torch.equal(got.cpu(), torch.from_numpy(want).float().to(dtype))
    if dtype != torch.float32:
        q, o = room(), room()
        q.copy_(s.rows(n, dtype=dtype))
        s.kv.attend(s.cache, seqs, q, out=o)
        near(o, None, s.ref.attend(s.table, [70, 31], begin, host(q.double()), 64 ** -0.5), dtype)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("block,dim", [(16, 64), (32, 256), (64, 128)])
def test_read(kind, dtype, block, dim):
    length = [200, 1, 64, 0, 95]
    s = Setup(length, block=block, dim=dim, kind=kind)
    s.fill()
    for new in ([200, 1, 64, 0, 95], [3, 0, 17, 0, 64], [0, 0, 0, 0, 1]):
        seqs, begin = s.seqs(length, new)
        got = s.kv.read(s.cache, seqs, dtype=dtype)
        for a, b in zip(got, s.ref.read(s.table, length, begin)):
            # codes times a power of two are exact in 32 bits: one rounding to the type
            assert torch.equal(a.cpu(), torch.from_numpy(b).float().to(dtype))
    length = [200, 1, 64, 95]
    keep = [0, 1, 2, 4]
    seqs = s.kv.Seqs(s.d_table[keep].contiguous(), torch.tensor(length, dtype=torch.int32, device="cuda"))
    got = s.kv.read(s.cache, seqs, dtype=dtype)
    for a, b in zip(got, s.ref.read(s.table[keep], length, np.arange(5))):
        assert torch.equal(a.cpu(), torch.from_numpy(b).float().to(dtype))


# ---- attention

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("block,dim,heads,group,dtype", [
    (16, 64, 2, 1, torch.bfloat16), (32, 128, 1, 4, torch.float16), (64, 128, 2, 8, torch.bfloat16),
    (64, 256, 1, 3, torch.float16), (16, 128, 1, 16, torch.bfloat16), (32, 64, 1, 21, torch.float16)])
def test_attend_token(kind, block, dim, heads, group, dtype):
    """One token of each sequence, lengths around every tile's end, none at all among them."""
    length = [1, 0, 15, 16, 17, 63, 64, 65, 127, 128, 257, 700, 1025]
    s = Setup(length, heads=heads, dim=dim, block=block, kind=kind)
    s.fill()
    seqs, begin = s.seqs(length)
    q = s.rows(len(length), heads * group, dtype)
    lse = torch.empty(len(length), heads * group, device="cuda")
    out = s.kv.attend(s.cache, seqs, q, lse=lse)
    near(out, lse, s.ref.attend(s.table, length, begin, host(q.double()), dim ** -0.5), dtype)
    assert not out[1].any()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("block,dim,heads,group,dtype", [
    (16, 64, 2, 1, torch.bfloat16), (32, 128, 1, 4, torch.float16), (64, 128, 1, 5, torch.bfloat16),
    (64, 256, 1, 2, torch.float16), (64, 64, 1, 12, torch.bfloat16)])
@pytest.mark.parametrize("new", [[1, 0, 5, 64, 0, 200, 33], [30, 1, 100, 190, 3, 300, 130]])
def test_attend_prompt(kind, block, dim, heads, group, dtype, new):
    """Rows that end their sequences, causal; more rows than tokens (rows that see nothing)."""
    length = [30, 1, 100, 190, 0, 300, 77]
    s = Setup(length, heads=heads, dim=dim, block=block, kind=kind)
    s.fill()
    seqs, begin = s.seqs(length, new)
    q = s.rows(int(begin[-1]), heads * group, dtype)
    lse = torch.empty(len(q), heads * group, device="cuda")
    out = s.kv.attend(s.cache, seqs, q, lse=lse)
    near(out, lse, s.ref.attend(s.table, length, begin, host(q.double()), dim ** -0.5), dtype)


@pytest.mark.parametrize("new", [None, [1, 1], [40, 3]])
def test_attend_long(new):
    """A long axis split over workgroups and joined."""
    length = [9000, 4100]
    s = Setup(length, heads=1, kind=INT8)
    s.fill()
    seqs, begin = s.seqs(length, new)
    q = s.rows(int(begin[-1]), 4)
    lse = torch.empty(len(q), 4, device="cuda")
    out = s.kv.attend(s.cache, seqs, q, lse=lse)
    near(out, lse, s.ref.attend(s.table, length, begin, host(q.double()), 128 ** -0.5), torch.bfloat16)


@pytest.mark.parametrize("new", [None, [300]])
@pytest.mark.parametrize("size", [0.01, 8.0])
def test_attend_sharp_and_flat(new, size):
    """Scores of hundreds, and weights that are all alike; values whose sizes differ from block
    to block by powers of two; a negative scale."""
    s = Setup([900], heads=1, block=16)
    for n in range(100, 901, 100):
        s.write([n], [100], size=2.0 ** ((n // 100 * 5) % 13 - 6))
    seqs, begin = s.seqs([900], new)
    for scale in (128 ** -0.5, -0.05):
        q = s.rows(int(begin[-1]), 2, size=size)
        out = s.kv.attend(s.cache, seqs, q, scale=scale)
        near(out, None, s.ref.attend(s.table, [900], begin, host(q.double()), scale), torch.bfloat16)


def test_attend_query_range():
    """Tiny and huge queries, a row of zeros, elements 2^20 apart."""
    s = Setup([130], heads=1, dim=64)
    s.fill()
    seqs, begin = s.seqs([130], [6])
    q = s.rows(6, 2)
    q[0], q[1], q[2] = 0, q[1] * 1e-30, q[2] * 2.0 ** -20
    q[3, :, 1:] *= 2.0 ** -20
    q[4] *= 1e30
    ref = host(q.double())
    out = s.kv.attend(s.cache, seqs, q, scale=0.1)
    want = s.ref.attend(s.table, [130], begin, ref, 0.1)
    keep = [0, 1, 2, 3, 5]
    near(out[keep], None, tuple(x[keep] for x in want), torch.bfloat16)
    assert torch.isfinite(out[4].float()).all()


@pytest.mark.parametrize("new", [None, [90, 7]])
def test_attend_blocks(new):
    """Lists of blocks: any subset, in any order, empty places, nothing at all."""
    length = [1000, 77]
    s = Setup(length, heads=2, block=32)
    s.fill()
    seqs, begin = s.seqs(length, new)
    n, keep = int(begin[-1]), 7
    blocks = np.full((n, 2, keep), -1, np.int32)
    for i in range(2):
        for row in range(begin[i], begin[i + 1]):
            last = (length[i] - (begin[i + 1] - begin[i]) + row - begin[i]) // 32
            for h in range(2):
                some = s.rng.permutation(last + 1)[:s.rng.integers(0, keep + 1)]
                at = s.rng.permutation(keep)[:len(some)]
                blocks[row, h, at] = some
    q = s.rows(n, 2 * 3)
    lse = torch.empty(n, 6, device="cuda")
    out = s.kv.attend(s.cache, seqs, q, blocks=torch.from_numpy(blocks).cuda(), lse=lse)
    near(out, lse, s.ref.attend(s.table, length, begin, host(q.double()), 128 ** -0.5, blocks), torch.bfloat16)


# ---- selection

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("block,dim,group,dtype", [(16, 64, 1, torch.bfloat16), (32, 128, 4, torch.float16),
                                                   (64, 256, 5, torch.bfloat16), (16, 128, 17, torch.float16)])
@pytest.mark.parametrize("keep,first,recent", [(1, 0, 1), (3, 1, 2), (9, 1, 2), (20, 0, 20), (33, 5, 3)])
def test_select(kind, block, dim, group, dtype, keep, first, recent):
    length = [block * 40 + 3, 1, 0, block * 9, block * 21 + block - 1]
    s = Setup(length, dim=dim, block=block, kind=kind)
    s.fill()
    for new in (None, [3, 1, 0, 2, 5]):
        seqs, begin = s.seqs(length, new)
        q = s.rows(int(begin[-1]), 2 * group, dtype)
        got = s.kv.select(s.cache, seqs, q, keep=keep, first=first, recent=recent)
        want = s.ref.select(s.table, length, begin, host(q.double()), keep, first, recent)
        assert np.array_equal(host(got), want)


def test_select_ties():
    """Equal scores: the lowest index.  A query of zeros ties all blocks; repeated keys some."""
    s = Setup([16 * 700], heads=1, dim=64, block=16)
    n = 16 * 700
    k = s.rows(n)
    k[16 * 20:16 * 600] = k[:16].repeat(580, 1, 1)
    seqs, begin = s.seqs([n], [n])
    s.kv.write(s.cache, seqs, k, k)
    s.ref.write(s.table, [n], begin, host(k.double()), host(k.double()))
    s.same()
    seqs, begin = s.seqs([n], [2])
    q = s.rows(2, 2)
    q[0] = 0
    for keep in (5, 300, 650):
        got = s.kv.select(s.cache, seqs, q, keep=keep, first=1, recent=1)
        assert np.array_equal(host(got), s.ref.select(s.table, [n], begin, host(q.double()), keep, 1, 1))


def test_select_feeds_attend():
    length = [2000, 640]
    s = Setup(length, block=32, kind=INT8)
    s.fill()
    seqs, begin = s.seqs(length, [3, 1])
    q = s.rows(4, 8)
    blocks = s.kv.select(s.cache, seqs, q, keep=10, first=1, recent=2)
    out = s.kv.attend(s.cache, seqs, q, blocks=blocks)
    near(out, None, s.ref.attend(s.table, length, begin, host(q.double()), 128 ** -0.5, host(blocks)), torch.bfloat16)


# ---- how it is called

def test_past_32_bits():
    """Blocks beyond 2^31 bytes of codes: the same results there as at the start."""
    kv = module()
    n_blocks, heads, dim, block = 36_000, 8, 128, 64  # 2.36 GB of keys, as much of values
    code = [torch.zeros((n_blocks, heads) + x, dtype=torch.uint8, device="cuda") for x in ((block, dim), (dim, block))]
    small = [torch.zeros((n_blocks, heads) + x, dtype=torch.int8, device="cuda") for x in ((), (), (dim,), ())]
    cache = kv.Cache(code[0], code[1], *small)
    length = torch.tensor([200], dtype=torch.int32, device="cuda")
    begin = torch.tensor([0, 200], dtype=torch.int64, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v, q = (torch.randn(200, 8, 128, generator=g, device="cuda").bfloat16() for _ in range(3))
    got = []
    for first in (0, n_blocks - 4):
        table = (first + torch.arange(4, device="cuda", dtype=torch.int32))[None].contiguous()
        seqs = kv.Seqs(table, length, begin=begin)
        kv.write(cache, seqs, k, v)
        one = kv.Seqs(table, length)
        got.append((kv.attend(cache, seqs, q), kv.attend(cache, one, q[-1:]), *kv.read(cache, seqs),
                    kv.select(cache, seqs, q, keep=2)))
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_wide_strides_past_32_bits():
    """A row's offset in elements beyond 2^31."""
    kv = module()
    s = Setup([64, 64], heads=1, dim=64)
    stride = (1 << 31) + 64
    space = torch.empty(stride + 4 * 64, dtype=torch.bfloat16, device="cuda")
    seqs, begin = s.seqs([64, 64], None)
    s.fill()
    q = space.as_strided((2, 4, 64), (stride, 64, 1))
    q.copy_(s.rows(2, 4))
    out = kv.attend(s.cache, seqs, q)
    assert torch.equal(out, kv.attend(s.cache, seqs, q.contiguous()))


def test_repeats_and_streams():
    """The same bits on every call, also on another stream than the tensors' own."""
    length = [5000, 77, 900]
    s = Setup(length)
    s.fill()
    for new in (None, [200, 5, 1]):
        seqs, begin = s.seqs(length, new)
        q = s.rows(int(begin[-1]), 8)
        want = s.kv.attend(s.cache, seqs, q)
        blocks = s.kv.select(s.cache, seqs, q, keep=5)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        for _ in range(5):
            assert torch.equal(s.kv.attend(s.cache, seqs, q), want)
            got = s.kv.attend(s.cache, seqs, q, stream=side)
            picked = s.kv.select(s.cache, seqs, q, keep=5, stream=side)
            side.synchronize()
            assert torch.equal(got, want) and torch.equal(picked, blocks)


def test_graph():
    """A step recorded and replayed on lengths and rows that change in place."""
    kv = module()
    s = Setup([400, 130], block=16, garbage=False)
    length = torch.tensor([300, 30], dtype=torch.int32, device="cuda")
    s.write([300, 30], [300, 30])
    seqs = kv.Seqs(s.d_table, length)
    k, v, q = s.rows(2), s.rows(2), s.rows(2, 8)
    status = kv.new_status()
    out, blocks = torch.empty_like(q), torch.empty(2, 2, 6, dtype=torch.int32, device="cuda")
    space = [kv.workspace(op, s.cache, seqs, q_heads=8, keep=6) for op in (kv.OP_ATTEND, kv.OP_SELECT)]

    def step():
        kv.write(s.cache, seqs, k, v, status=status, check=False)
        kv.select(s.cache, seqs, q, keep=6, out=blocks, workspace=space[1], status=status, check=False)
        kv.attend(s.cache, seqs, q, blocks=blocks, out=out, workspace=space[0], status=status, check=False)

    n = [300, 30]
    graph = torch.cuda.CUDAGraph()
    length.add_(1)
    step()  # before the recording, as a program warms up; its token is written again below
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    length.sub_(1)
    for i in range(40):
        length.add_(1)
        n = [x + 1 for x in n]
        k.copy_(s.rows(2)), v.copy_(s.rows(2)), q.copy_(s.rows(2, 8))
        if i == 0:
            # the warm-up's token is in the reference only as what it left: a scale
            for name in ("k_code", "v_code", "k_exp", "v_exp", "mean_code", "mean_exp"):
                getattr(s.ref, name)[...] = host(getattr(s.cache, name))
        graph.replay()
        s.ref.write(s.table, n, np.arange(3), host(k.double()), host(v.double()))
        want = s.ref.select(s.table, n, np.arange(3), host(q.double()), 6, 1, 1)
        assert np.array_equal(host(blocks), want)
        near(out, None, s.ref.attend(s.table, n, np.arange(3), host(q.double()), 128 ** -0.5, want), torch.bfloat16)
    assert status.item() == 0


def test_empty_calls():
    kv = module()
    s = Setup([10])
    empty = torch.empty(0, 2, 128, dtype=torch.bfloat16, device="cuda")
    seqs, _ = s.seqs([10], [0])
    none = kv.Seqs(s.d_table[:0], torch.empty(0, dtype=torch.int32, device="cuda"))
    for x in (seqs, none):
        kv.write(s.cache, x, empty, empty)
        kv.read(s.cache, x)
        assert kv.attend(s.cache, x, empty).numel() == 0
        picked = kv.select(s.cache, x, empty, keep=3)
        assert kv.attend(s.cache, x, empty, blocks=picked).numel() == 0


# ---- refusals found on the device

def raised(s, call):
    status = s.kv.new_status()
    call(status)
    torch.cuda.synchronize()
    return status.item()


@pytest.mark.parametrize("new", [None, [20, 7]])
@pytest.mark.parametrize("fault", ["none", "entry", "negative_entry", "length", "negative_length", "begin", "end",
                                   "falling", "most_new"])
def test_data_errors(new, fault):
    """Each is MP_EINVAL on the status word of every operator that meets it."""
    if new is None and fault in ("begin", "end", "falling", "most_new"):
        pytest.skip("no begin in this form")
    s = Setup([300, 7], block=32, garbage=False)
    s.fill()
    table, length = s.d_table.clone(), torch.tensor([300, 7], dtype=torch.int32, device="cuda")
    begin = None if new is None else torch.tensor([0, 20, 27], dtype=torch.int64, device="cuda")
    tokens = 2 if new is None else 27
    more = {"most_new": 20} if new else {}
    if fault == "entry":
        table[0, 9] = s.cache.n_blocks
    elif fault == "negative_entry":
        table[1, 0] = -1
    elif fault == "length":
        length[1] = 400
    elif fault == "negative_length":
        length[0] = -5
    elif fault == "begin":
        begin[0] = 1
    elif fault == "end":
        begin[2] = 28
    elif fault == "falling":
        begin[1] = 28
    elif fault == "most_new":
        more = {"most_new": 19}
    seqs = s.kv.Seqs(table, length, begin=begin, tokens=tokens, longest=320, **more)
    want = 0 if fault == "none" else -1
    k, q = s.rows(tokens), s.rows(tokens, 4)
    assert raised(s, lambda st: s.kv.read(s.cache, seqs, status=st, check=False)) == want
    assert raised(s, lambda st: s.kv.attend(s.cache, seqs, q, status=st, check=False)) == want
    if "entry" not in fault:  # a selection reads no table entry that it does not score
        assert raised(s, lambda st: s.kv.select(s.cache, seqs, q, keep=4, status=st, check=False)) == want
    assert raised(s, lambda st: s.kv.write(s.cache, seqs, k, k, status=st, check=False)) == want


def test_data_errors_of_lists_and_rows():
    s = Setup([300], block=32, garbage=False)
    s.fill()
    seqs, _ = s.seqs([300])
    q = s.rows(1, 4)
    for bad in (10, -2, 1 << 30):
        blocks = torch.tensor([[[0, bad], [1, 2]]], dtype=torch.int32, device="cuda")
        assert raised(s, lambda st: s.kv.attend(s.cache, seqs, q, blocks=blocks, status=st, check=False)) == -1
    # more rows than tokens cannot be written or read
    seqs, _ = s.seqs([3], [5])
    k = s.rows(5)
    assert raised(s, lambda st: s.kv.write(s.cache, seqs, k, k, status=st, check=False)) == -1
    assert raised(s, lambda st: s.kv.read(s.cache, seqs, status=st, check=False)) == -1
    with pytest.raises(s.kv.PlanError):
        s.kv.write(s.cache, seqs, k, k)


def test_argument_errors():
    s = Setup([100], heads=2, dim=64, block=16)
    seqs, _ = s.seqs([100])
    k, q, kv = s.rows(1), s.rows(1, 4), s.kv
    c = s.cache
    with pytest.raises(ValueError):
        kv.write(c, seqs, k[..., :32], k)
    with pytest.raises(ValueError):
        kv.write(c, seqs, k.expand(2, 2, 64), k)
    with pytest.raises(TypeError):
        kv.write(c, seqs, k.double(), k)
    with pytest.raises(TypeError):
        kv.attend(c, seqs, q.float())
    with pytest.raises(TypeError):
        kv.attend(c, seqs, q.cpu())
    with pytest.raises(ValueError):
        kv.attend(c, seqs, torch.empty(1, 4, 128, dtype=q.dtype, device="cuda")[..., ::2])
    with pytest.raises(kv.PlanError):
        kv.attend(c, seqs, s.rows(1, 3))  # 3 query heads over 2
    with pytest.raises(TypeError):
        kv.attend(c, seqs, q, out=torch.empty_like(q, dtype=torch.float16))
    with pytest.raises(ValueError):
        kv.attend(c, seqs, q, blocks=torch.zeros(1, 1, 3, dtype=torch.int32, device="cuda"))
    with pytest.raises(kv.PlanError):
        kv.select(c, seqs, q, keep=3, first=2, recent=2)
    with pytest.raises(kv.PlanError):
        kv.select(c, seqs, q, keep=3, first=1, recent=0)
    with pytest.raises(ValueError):
        kv.Cache(c.k_code, c.v_code, c.k_exp, c.v_exp, c.mean_code[:, :, :32], c.mean_exp)
    with pytest.raises(ValueError):
        kv.Cache(c.k_code, c.v_code, c.k_exp, c.v_exp, c.mean_code, c.mean_exp, kind=2)
    with pytest.raises(kv.PlanError):
        kv.write(kv.new_cache(4, 2, 96, block=16), kv.Seqs(s.d_table, seqs.length), k[..., :1].expand(1, 2, 96).contiguous(),
                 k[..., :1].expand(1, 2, 96).contiguous())
    with pytest.raises(ValueError):
        kv.Seqs(s.d_table, seqs.length, tokens=3)


def test_select_of_very_long_sequences():
    """More blocks than scores fit on chip: the same selection from a workspace, which is asked for."""
    blocks = 17_000
    s = Setup([16 * 40], heads=2, dim=64, block=16)
    s.fill()
    # a table that names the same few blocks over and over
    table = np.resize(s.table[:1, :40], (1, blocks)).astype(np.int64)
    length = [blocks * 16 - 5]
    s.table = table
    seqs = s.kv.Seqs(torch.from_numpy(table.astype(np.int32)).cuda(),
                     torch.tensor(length, dtype=torch.int32, device="cuda"),
                     begin=torch.tensor([0, 3], dtype=torch.int64, device="cuda"), tokens=3)
    q = s.rows(3, 6)
    assert s.kv.workspace_size(s.kv.OP_SELECT, s.cache, seqs, q_heads=6, keep=50) > 0
    got = s.kv.select(s.cache, seqs, q, keep=50, first=2, recent=3)
    assert np.array_equal(host(got), s.ref.select(table, length, [0, 3], host(q.double()), 50, 2, 3))
    with pytest.raises(s.kv.PlanError):
        s.kv.select(s.cache, seqs, q, keep=50, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("block", [16, 64])
def test_attend_long_prompt(kind, block):
    """Prompts of over a thousand tokens beside short and empty ones and one that sees nothing
    of its first rows: the form for the longest pieces."""
    length, new = [1100, 300, 5, 0, 640], [1100, 20, 9, 3, 640]
    s = Setup(length, heads=1, block=block, kind=kind)
    s.fill()
    seqs, begin = s.seqs(length, new)
    q = s.rows(int(begin[-1]), 4)
    lse = torch.empty(len(q), 4, device="cuda")
    out = s.kv.attend(s.cache, seqs, q, lse=lse)
    near(out, lse, s.ref.attend(s.table, length, begin, host(q.double()), 128 ** -0.5), torch.bfloat16)
    out = s.kv.attend(s.cache, seqs, q * 20, scale=-0.3)
    near(out, None, s.ref.attend(s.table, length, begin, host((q * 20).double()), -0.3), torch.bfloat16)


@pytest.mark.parametrize("scale", [0.0, 1e-30])
@pytest.mark.parametrize("new", [None, [6], [200], [1030]])
def test_attend_scale_of_nothing(scale, new):
    """Equal weights: the mean of what is seen, in every form."""
    s = Setup([1030], heads=1, dim=128)
    s.fill()
    seqs, begin = s.seqs([1030], new)
    q = s.rows(int(begin[-1]), 4)
    out = s.kv.attend(s.cache, seqs, q, scale=scale)
    near(out, None, s.ref.attend(s.table, [1030], begin, host(q.double()), scale), torch.bfloat16)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,new", [(64, 16), (128, 70), (64, 300), (128, 1100)])
def test_attend_ignores_sizes_of_later_blocks(kind, dim, new):
    """Values that grow by 2^13 a block: what a row does not see yet, however large, costs it no
    bits.  The bound is that of the blocks it sees."""
    block, group, blocks = 16, 4, 70
    s = Setup([block * blocks], heads=1, dim=dim, block=block, kind=kind)
    for b in range(blocks):
        n = b * block
        seqs, begin = s.seqs([n + block], [block])
        k, v = s.rows(block), s.rows(block, size=2.0 ** (13 * (b % 8) - 50))
        s.kv.write(s.cache, seqs, k, v)
        s.ref.write(s.table, [n + block], begin, host(k.double()), host(v.double()))
    for length in (block * 8 - 3, block * blocks):
        seqs, begin = s.seqs([length], [min(new, length)])
        q = s.rows(int(begin[-1]), group)
        out = s.kv.attend(s.cache, seqs, q)
        ref, ref_lse, mass, delta, floor = s.ref.attend(s.table, [length], begin, host(q.double()), dim ** -0.5)
        top = np.maximum.accumulate(s.ref.v_exp[s.table[0, :blocks], 0].astype(float))
        last = length - len(q) + np.arange(len(q))
        largest = (448.0 if kind == E4M3 else 127.0) * 2.0 ** top[last // block]
        floor = np.broadcast_to(((last + 1) * largest)[:, None], floor.shape)
        near(out, None, (ref, ref_lse, mass, delta, floor), torch.bfloat16)


def test_inputs_that_share_places():
    """One head's rows for all heads, one token's for all: read as they are."""
    s = Setup([70], heads=3, dim=64, block=32, garbage=False)
    seqs, begin = s.seqs([70], [70])
    k, v = s.rows(70, 1).expand(70, 3, 64), s.rows(1, 3).expand(70, 3, 64)
    s.kv.write(s.cache, seqs, k, v)
    s.ref.write(s.table, [70], begin, host(k.double()), host(v.double()))
    s.same()
    s.same_codes([70])
    q = s.rows(1, 1).expand(70, 6, 64)
    near(s.kv.attend(s.cache, seqs, q), None, s.ref.attend(s.table, [70], begin, host(q.double()), 64 ** -0.5),
         torch.bfloat16)


def test_refusals_of_places():
    """Outputs, tables, workspaces and lists whose memory is not what the call would take it for."""
    s = Setup([100, 50], heads=2, dim=64, block=16)
    seqs, _ = s.seqs([100, 50])
    q, kv, c = s.rows(2, 4), s.kv, s.cache
    for out in (torch.empty(1, 4, 64, dtype=q.dtype, device="cuda").expand(2, 4, 64),
                torch.empty(2, 1, 64, dtype=q.dtype, device="cuda").expand(2, 4, 64)):
        with pytest.raises(kv.PlanError):
            kv.attend(c, seqs, q, out=out)
        with pytest.raises(kv.PlanError):
            kv.read(c, seqs, out=(out[:, :2], torch.empty(2, 2, 64, dtype=q.dtype, device="cuda")))
    with pytest.raises(ValueError):
        kv.Seqs(s.d_table[:1].expand(2, -1), seqs.length)
    need = kv.workspace_size(kv.OP_ATTEND, c, seqs, q_heads=4, keep=4)
    with pytest.raises(ValueError):
        kv.attend(c, seqs, q, workspace=torch.empty(2 * (need + 64), dtype=torch.uint8, device="cuda")[::2])
    with pytest.raises(ValueError):
        kv.attend(c, seqs, q, blocks=torch.empty(2, 2, 0, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        kv.attend(c, seqs, q, status=torch.zeros(0, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("new", [None, [3]])
@pytest.mark.parametrize("blocks", [66, 258, 259, 515, 1026, 1027, 1028, 2500])
def test_select_of_many_blocks(blocks, new):
    """Around the numbers of blocks at which the selection changes its form, many ties among them."""
    s = Setup([16 * 50], heads=2, dim=64, block=16)
    s.fill()
    table = np.resize(s.table[:1, :50], (1, blocks)).astype(np.int64)
    length = [blocks * 16 - 5]
    begin = np.array([0, 1 if new is None else new[0]])
    seqs = s.kv.Seqs(torch.from_numpy(table.astype(np.int32)).cuda(),
                     torch.tensor(length, dtype=torch.int32, device="cuda"),
                     begin=None if new is None else torch.from_numpy(begin).cuda(), tokens=int(begin[-1]))
    q = s.rows(int(begin[-1]), 6)
    for keep, first, recent in ((1, 0, 1), (2, 1, 1), (17, 2, 3), (min(64, blocks - 1), 1, 2), (blocks - 1, 0, 1)):
        got = s.kv.select(s.cache, seqs, q, keep=keep, first=first, recent=recent)
        assert np.array_equal(host(got), s.ref.select(table, length, begin, host(q.double()), keep, first, recent))
