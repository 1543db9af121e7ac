"""The forms of the 8-bit key/value cache's kernels that only larger calls take: over 256 workgroups
of few rows, lists of blocks longer than a chunk, groups of over 16 query heads, heads of 256, and
batches whose search for a row's sequence takes more than one turn.  Against the definition."""
import numpy as np
import pytest
import torch

from gpu_util import host
from test_gpu_kv import KINDS, Setup, near

pytestmark = pytest.mark.gpu


def lists(s, length, begin, keep):
    """A list for every row and key head: some of the blocks it sees, in any order, empty places."""
    out = np.full((int(begin[-1]), s.heads, keep), -1, np.int32)
    for i in range(len(length)):
        n = begin[i + 1] - begin[i]
        for row in range(begin[i], begin[i + 1]):
            last = length[i] - n + row - begin[i]
            for h in range(s.heads if last >= 0 else 0):
                some = s.rng.permutation(last // s.block + 1)[:s.rng.integers(keep // 2, keep + 1)]
                out[row, h, s.rng.permutation(keep)[:len(some)]] = some
    return out


def attended(s, length, new, group, keep=0, dtype=torch.bfloat16):
    seqs, begin = s.seqs(length, new, **({} if new is None else {"most_new": max(new)}))
    q = s.rows(int(begin[-1]), s.heads * group, dtype)
    lse = torch.empty(len(q), s.heads * group, device="cuda")
    blocks = lists(s, length, begin, keep) if keep else None
    out = s.kv.attend(s.cache, seqs, q, lse=lse, blocks=None if blocks is None else torch.from_numpy(blocks).cuda())
    near(out, lse, s.ref.attend(s.table, length, begin, host(q.double()), s.dim ** -0.5, blocks), dtype)


def batch(n, most, seed):
    """Lengths of n sequences, some of one token, some of none, one of `most`."""
    length = np.random.default_rng(seed).integers(2, most, n)
    length[::9], length[4::11], length[n // 2] = 1, 0, most
    return [int(x) for x in length]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,block", [(64, 16), (64, 64), (128, 32), (128, 64)])
@pytest.mark.parametrize("form", ["one", "several", "list", "lists"])
def test_many_workgroups_of_few_rows(kind, dim, block, form):
    """70 sequences of 4 key heads: over 256 workgroups."""
    length = batch(70, 600, dim + block)
    s = Setup(length, heads=4, dim=dim, block=block, kind=kind)
    s.fill()
    new = [min(n, 1 + i % 5) for i, n in enumerate(length)] if form in ("several", "lists") else None
    attended(s, length, new, 3, keep=6 if "list" in form else 0)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,block,keep,group", [(128, 64, 17, 4), (128, 64, 64, 2), (64, 32, 33, 5), (64, 64, 40, 17),
                                                  (128, 16, 150, 21), (256, 64, 5, 3), (256, 32, 40, 2)])
@pytest.mark.parametrize("new", [None, [3, 2]])
def test_long_lists(kind, dim, block, keep, group, new):
    """Lists of more blocks than one workgroup takes, some of them in part: joined."""
    length = [5003, 900]
    s = Setup(length, dim=dim, block=block, kind=kind)
    s.fill()
    attended(s, length, new, group, keep=keep)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new", [[5, 1, 3, 0, 2], [40, 1, 90, 0, 3]])
@pytest.mark.parametrize("group", [1, 4])
def test_heads_of_256(kind, new, group):
    length = [1500, 1, 90, 0, 700]
    s = Setup(length, heads=1, dim=256, block=32, kind=kind)
    s.fill()
    attended(s, length, new, group, dtype=torch.float16)


@pytest.mark.parametrize("n", [63, 64, 65, 300])
@pytest.mark.parametrize("most_new", [3, 60])
def test_many_sequences_with_pieces(n, most_new):
    """Pieces of 63-300 sequences, empty ones among them: written, read, attended to (rows, tiles),
    selected from."""
    length = batch(n, 150, n)
    s = Setup(length, heads=2, dim=64, block=16)
    new = [min(x, (i * 7) % (most_new + 1)) for i, x in enumerate(length)]
    start = [a - b for a, b in zip(length, new)]
    s.write(start, start)
    s.write(length, new, size=4.0)
    s.same()
    s.same_codes(length)
    seqs, begin = s.seqs(length, new)
    for a, b in zip(s.kv.read(s.cache, seqs), s.ref.read(s.table, length, begin)):
        assert torch.equal(a.cpu(), torch.from_numpy(b).float().bfloat16())
    attended(s, length, new, 4)
    q = s.rows(int(begin[-1]), 4)
    got = s.kv.select(s.cache, seqs, q, keep=4, first=1, recent=1)
    assert np.array_equal(host(got), s.ref.select(s.table, length, begin, host(q.double()), 4, 1, 1))


def test_long_prompts_of_many_sequences():
    """The form for the longest pieces where over 64 sequences share a launch."""
    length = [1100] + [40 + i % 90 for i in range(70)] + [0, 1, 300]
    new = [1100] + [min(n, i % 70) for i, n in enumerate(length[1:])]
    s = Setup(length, heads=1, block=64)
    s.fill()
    attended(s, length, new, 4)
