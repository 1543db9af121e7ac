"""Means of a cache at a multiple of 8 bytes that is none of 16, which the contract allows: written and
selected from as anywhere else."""
import numpy as np
import pytest
import torch

from gpu_util import host
from test_gpu_kv import Setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,block,new", [(64, 16, None), (128, 32, [3, 2]), (256, 64, None)])
def test_means_at_eight_bytes(dim, block, new):
    length = [block * 30 + 5, block * 12]
    s = Setup(length, dim=dim, block=block)
    c = s.cache
    space = torch.zeros(c.mean_code.numel() + 32, dtype=torch.int8, device="cuda")
    first = 8 + (-space.data_ptr()) % 16
    means = space[first:first + c.mean_code.numel()].view(c.mean_code.shape)
    assert means.data_ptr() % 16 == 8
    means.copy_(c.mean_code)
    s.cache = s.kv.Cache(c.k_code, c.v_code, c.k_exp, c.v_exp, means, c.mean_exp, kind=s.kind)
    s.fill()
    s.same()
    seqs, begin = s.seqs(length, new)
    q = s.rows(int(begin[-1]), 6)
    got = s.kv.select(s.cache, seqs, q, keep=7, first=1, recent=2)
    assert np.array_equal(host(got), s.ref.select(s.table, length, begin, host(q.double()), 7, 1, 2))
