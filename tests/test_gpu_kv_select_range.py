"""Selection of blocks at the ends of the ranges of queries and keys: scores are exact, so the blocks are
those of the definition in 64 bits."""
import numpy as np
import pytest
import torch

from gpu_util import host
from test_gpu_kv import KINDS, Setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new", [None, [5]])
@pytest.mark.parametrize("keys", [-85, -60, 0, 60, 110])
@pytest.mark.parametrize("queries", [-130, -120, -60, 0, 60, 120])
def test_sizes_of_queries_and_keys(kind, new, keys, queries):
    """Keys about 2^keys, their blocks within 2^6 of each other, queries about 2^queries, heads alike: from
    subnormal to nearly the largest."""
    length = [16 * 60 + 3]
    s = Setup(length, heads=2, dim=64, block=16, kind=kind)
    block = torch.arange(length[0]) // 16
    k = s.rows(length[0]).cpu().double() * 2.0 ** (keys + (block * 5 % 7)[:, None, None])
    k = k.float()
    seqs, begin = s.seqs(length, length)
    s.kv.write(s.cache, seqs, k.cuda(), k.cuda())
    s.ref.write(s.table, length, begin, k.double().numpy(), k.double().numpy())
    s.same()
    seqs, begin = s.seqs(length, new)
    q = (s.rows(int(begin[-1]), 6).double() * 2.0 ** queries).bfloat16()
    assert q.abs().max() > 0 and torch.isfinite(q).all()
    for keep in (4, 20, 59):
        got = s.kv.select(s.cache, seqs, q, keep=keep, first=1, recent=1)
        assert np.array_equal(host(got), s.ref.select(s.table, length, begin, host(q.double()), keep, 1, 1))


@pytest.mark.parametrize("new", [None, [5]])
def test_heads_of_different_sizes(new):
    """Query heads of one key head 2^15 apart, one of them zeros; 21 heads, over one instruction's columns."""
    length = [16 * 80]
    s = Setup(length, heads=1, dim=128, block=16)
    s.fill()
    seqs, begin = s.seqs(length, new)
    for group in (3, 21):
        q = s.rows(int(begin[-1]), group)
        q *= 2.0 ** (-15.0 * (torch.arange(group, device="cuda") % 4))[:, None]
        q[:, group // 2] = 0
        got = s.kv.select(s.cache, seqs, q, keep=9, first=1, recent=1)
        assert np.array_equal(host(got), s.ref.select(s.table, length, begin, host(q.double()), 9, 1, 1))
