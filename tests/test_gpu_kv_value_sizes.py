"""Attention over the 8-bit key/value cache whose values differ widely in size from block to block:
what a weight loses is small beside the largest contribution to its row, whichever block that is of."""
import numpy as np
import pytest
import torch

from gpu_util import host
from kv_defs import LIMIT
from test_gpu_kv import HALF_STEP, KINDS, LEAST_STEP, Setup

pytestmark = pytest.mark.gpu

LENGTH = 1100
FORMS = [pytest.param(None, 128, 64, id="one"), pytest.param(None, 128, 32, id="one32"),
         pytest.param("list", 64, 16, id="list"), pytest.param("list", 128, 64, id="list64"),
         pytest.param([6], 128, 16, id="several"), pytest.param([200], 64, 16, id="tiles64"),
         pytest.param([150], 256, 32, id="tiles256"), pytest.param([LENGTH], 128, 64, id="pair"),
         pytest.param([LENGTH], 128, 16, id="pair16")]


def definition(s, q, scale):
    """(out, mass, delta, reach) of queries q [rows, dim], the last tokens of the LENGTH: attention in 64
    bits; the weighted mean of |v|; the largest sum of |scale q k|; and the places seen times
    the largest |weight * value| that codes can stand for, over the sum of weights."""
    pages = s.table[0][:(LENGTH + s.block - 1) // s.block]
    k, v = (x[:LENGTH] for x in s.ref.values(pages, 0))
    size = LIMIT[s.kind] * 2.0 ** np.repeat(s.ref.v_exp[pages, 0].astype(float), s.block)[:LENGTH]
    place = LENGTH - len(q) + np.arange(len(q))
    hidden = np.arange(LENGTH) > place[:, None]
    x = scale * (q @ k.T)
    x[hidden] = -np.inf
    w = np.exp(x - x.max(1, keepdims=True))
    w /= w.sum(1, keepdims=True)
    delta = np.where(hidden, 0.0, scale * (np.abs(q) @ np.abs(k.T))).max(1)
    return w @ v, w @ np.abs(v), delta, (place + 1) * (w * size).max(1)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new,dim,block", FORMS)
@pytest.mark.parametrize("grown", [8, 20, 45, 200])
@pytest.mark.parametrize("where", ["first", "middle", "last", "steps"])
def test_one_size_above_the_others(kind, new, dim, block, grown, where):
    """Values 2^grown times the others' in some blocks, whose scores are lower by about as many powers of
    two (their contributions are alike) or by 24 more (the others' count).

    Scores: as everywhere, `dim` products and a few roundings of 2^-24 of the sum of |products|.  A
    weight has 11 bits, in 16-bit floats whose steps end at 2^-24; the largest contribution's weight is
    between 2^4 and 2^15 (sizes that differ by no more than 2^10 need not be told apart, a power of
    two is lost to whole exponents), so each is off by 2^-29 of what the largest contribution may be."""
    s = Setup([LENGTH], heads=1, dim=dim, block=block, kind=kind)
    of = torch.arange(LENGTH) // block
    count = int(of[-1]) + 1
    # "steps": a size for every block, in eight steps up to the largest
    part = {"first": of < 2, "middle": (of >= count // 2) & (of < count // 2 + 2), "last": of >= count - 2,
            "steps": of * 8 // count / 7}[where].double()
    scale = 2.0 ** -4
    for more in (0, 24):
        k = s.rows(LENGTH, 1).cpu() * 0.25
        # the first element's part of a score: 256 powers of two, less what is said above
        k[:, 0, 0] = 16.0 - part * (grown + more) / 16
        v = (s.rows(LENGTH, 1).cpu().double() * 2.0 ** (part * grown - 80)[:, None, None]).bfloat16()
        seqs, begin = s.seqs([LENGTH], [LENGTH])
        s.kv.write(s.cache, seqs, k.cuda(), v.cuda())
        s.ref.write(s.table, [LENGTH], begin, k.double().numpy(), v.double().numpy())

        seqs, begin = s.seqs([LENGTH], None if new == "list" else new)
        q = s.rows(int(begin[-1]), 1)[:, 0]
        q[:, 0] = 16.0 * 0.6931471805599453 / scale
        blocks = torch.arange(count, dtype=torch.int32, device="cuda")[None, None] if new == "list" else None
        out = s.kv.attend(s.cache, seqs, q[:, None].expand(-1, 4, -1), scale=scale, blocks=blocks)
        ref, mass, delta, reach = definition(s, host(q.double()), scale)
        score = ((dim + 8) * 2.0 ** -24 * delta)[:, None]
        bound = HALF_STEP[torch.bfloat16] * np.abs(ref) + (2.0 ** -11 + 2.0 ** -20 + 2.5 * score) * mass * 1.01
        bound += 2.0 ** -29 * reach[:, None] + LEAST_STEP[torch.bfloat16]
        off = np.abs(host(out.double()) - ref[:, None])
        assert np.all(off <= bound[:, None]), (more, np.nanmax(off / bound[:, None]))
