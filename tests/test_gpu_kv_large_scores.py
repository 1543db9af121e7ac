"""Attention over the 8-bit key/value cache where scores are large: successive tiles whose
scores differ by one power of two of a weight, and scores whose 32-bit steps are wider than
the weights' whole range.  Every form, against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from gpu_util import host
from test_gpu_kv import HALF_STEP, KINDS, LEAST_STEP, Setup

pytestmark = pytest.mark.gpu

LENGTH = 1100
SCALE = float(np.float32(math.log(2.0)))  # scores are counted in powers of two
# (rows of the sequence, heads' dim, block): one token, a list of blocks, a few tokens, tiles of rows for heads of
# 64 and 256, and the form for the longest pieces of heads of 128
FORMS = [pytest.param(None, 128, 64, id="one"), pytest.param("list", 64, 16, id="list"),
         pytest.param([6], 128, 16, id="several"), pytest.param([200], 64, 16, id="tiles64"),
         pytest.param([150], 256, 64, id="tiles256"), pytest.param([LENGTH], 128, 64, id="pair"),
         pytest.param([LENGTH], 128, 16, id="pair16")]


def definition(s, q, scale):
    """(out, mass, largest) of queries q [rows, dim], the last tokens of the LENGTH: attention in 64 bits,
    the weighted mean of |v|, and the places seen times the largest value that codes can stand for."""
    pages = s.table[0][:(LENGTH + s.block - 1) // s.block]
    k, v = (x[:LENGTH] for x in s.ref.values(pages, 0))
    x = scale * (q @ k.T)
    place = LENGTH - len(q) + np.arange(len(q))
    x[np.arange(LENGTH) > place[:, None]] = -np.inf
    w = np.exp(x - x.max(1, keepdims=True))
    w /= w.sum(1, keepdims=True)
    largest = (448.0 if s.kind == 0 else 127.0) * 2.0 ** float(s.ref.v_exp[pages, 0].max())
    return w @ v, w @ np.abs(v), (place + 1) * largest


def check(out, want, part, step=2.0 ** -40):
    """`part`: how far a weight may be off by its score's roundings.  The others: its own to 11 bits
    and in steps of `step` of the largest, the sums', the result's."""
    ref, mass, largest = want
    bound = HALF_STEP[torch.bfloat16] * np.abs(ref) + (2.0 ** -11 + 2.0 ** -20 + 2.1 * part) * mass * 1.01
    bound += step * largest[:, None] + LEAST_STEP[torch.bfloat16]
    off = np.abs(host(out.double()) - ref[:, None])
    assert np.all(off <= bound[:, None]), np.nanmax(off / bound[:, None])


def filled(kind, dim, block, first, second, size):
    """LENGTH tokens: keys with these two first elements, values of these sizes."""
    s = Setup([LENGTH], heads=1, dim=dim, block=block, kind=kind)
    k = torch.zeros(LENGTH, 1, dim)
    k[:, 0, 0], k[:, 0, 1] = first, second
    v = (torch.from_numpy(s.rng.standard_normal((LENGTH, 1, dim))) * size[:, None, None]).bfloat16()
    seqs, begin = s.seqs([LENGTH], [LENGTH])
    s.kv.write(s.cache, seqs, k.bfloat16().cuda(), v.cuda())
    s.ref.write(s.table, [LENGTH], begin, k.double().numpy(), v.double().numpy())
    return s


def attended(s, new, first, second, scale):
    """(out, the definition's results) of queries with these two first elements, four heads of each row."""
    listed = new == "list"
    seqs, begin = s.seqs([LENGTH], None if listed else new)
    q = torch.zeros(int(begin[-1]), s.dim)
    q[:, 0], q[:, 1] = first, second
    q = q.bfloat16()
    assert float(q[0, 0]) == first and float(q[0, 1]) == second
    blocks = None
    if listed:
        blocks = torch.arange((LENGTH + s.block - 1) // s.block, dtype=torch.int32, device="cuda")[None, None]
    out = s.kv.attend(s.cache, seqs, q.cuda()[:, None].expand(-1, 4, -1), scale=scale, blocks=blocks)
    return out, definition(s, q.double().numpy(), scale)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new,dim,block", FORMS)
@pytest.mark.parametrize("power", [15, 16, 17, 18, 19, 20, 22])
def test_tiles_one_power_apart(kind, new, dim, block, power):
    """Scores of tile i (64 tokens): 2^power + i or -2^power + i powers of two.  The maximum grows by
    one a tile.

    The products are exact; of a score three roundings remain (its factor's two, its own) and one
    of a chunk's logarithm, 2^-24 of it each, in powers of two.  The factor's is the same for all
    scores, which are 17 apart."""
    s = filled(kind, dim, block, 64.0, torch.arange(LENGTH) // 64, torch.ones(LENGTH))
    for sign in (1, -1):
        out, want = attended(s, new, sign * 2.0 ** power / 64, 1.0, SCALE)
        check(out, want, 2.0 ** (2 * 2.0 ** (power - 24) + 2.0 ** -16) - 1)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new,dim,block", FORMS)
@pytest.mark.parametrize("lower", [False, True])
def test_equal_huge_scores(kind, new, dim, block, lower):
    """Equal scores, with values of other sizes from block to block: the plain mean of what is seen.
    With `lower`, every third block's scores are half as far from zero: one sort alone counts.

    Equal scores are rounded alike, so their weights are equal; the others are 2^20 powers apart."""
    token = torch.arange(LENGTH)
    first = torch.where((token // block % 3 == 1) & lower, 32.0, 64.0)
    s = filled(kind, dim, block, first, 0.0, 2.0 ** (-3.0 * (token // block % 4)))
    for power in (21, 24, 25, 26, 28, 40):
        for part in (1.0, 1.2421875, -1.0, -1.2421875):
            out, want = attended(s, new, part * 2.0 ** power / 64, 0.0, SCALE)
            check(out, want, 0.0)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new,dim,block", FORMS)
def test_huge_scores_of_values_apart(kind, new, dim, block):
    """The same with sizes too far apart to share one exponent: weights end in steps of 2^-29 of what the
    largest contribution may be."""
    token = torch.arange(LENGTH)
    first = torch.where(token // block % 3 == 1, 32.0, 64.0)
    s = filled(kind, dim, block, first, 0.0, 2.0 ** (-9.0 * (token // block % 4)))
    for power in (12, 18, 24, 25, 28, 40):
        for part in (1.2421875, -1.2421875):
            out, want = attended(s, new, part * 2.0 ** power / 64, 0.0, SCALE)
            check(out, want, 2.0 ** (2 * 2.0 ** (power - 24) + 2.0 ** -16) - 1 if power < 21 else 0.0, 2.0 ** -29)
