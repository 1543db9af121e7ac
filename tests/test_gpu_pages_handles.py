"""What the handles of the blocks for requests hold after a call, and what is free in a pool."""
import numpy as np
import pytest
import torch

from gpu_util import dev, host
from test_gpu_pages import Setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [3, 2000])
def test_a_step_has_the_lengths(n):
    """Those that its calls read, wherever the call put them: in place, or in a tensor of the caller's."""
    s = Setup([20] * n, block=16, width=8)

    def all_are(lengths, value):
        return bool((lengths == value).all())

    step = s.extend([1] * n)
    assert all_are(step.length, 21) and all_are(s.length, 21)
    apart = torch.zeros(n, dtype=torch.int32, device="cuda")
    step = s.extend([2] * n, length_out=apart)
    assert all_are(step.length, 23) and all_are(s.length, 21)
    own = s.pages.new_step(n, 2 * n)
    got = s.pages.extend(s.pool, s.table, s.length, dev(np.full(n, 2), torch.int32), block=16, step=own,
                         length_out=own.length)
    assert got is own and all_are(own.length, 23) and all_are(s.length, 21)


def test_what_is_free():
    """The ids from the counter on are the blocks that no sequence holds, after any steps; those before it are not
    told apart."""
    rng = np.random.default_rng(2)
    s = Setup([int(x) for x in rng.integers(0, 100, 40)], block=16, width=30, spare=300)
    everything = np.sort(host(s.pool.ids))
    for _ in range(8):
        s.release(rng.random(40) < 0.4)
        s.extend(rng.integers(0, 60, 40).tolist())
        length, table, used = host(s.length), host(s.table), int(s.pool.used.item())
        held = [b for n, row in zip(length, table) for b in row[:(n + 15) // 16]]
        assert used == len(held)
        assert np.array_equal(np.sort(np.concatenate([held, host(s.pool.ids)[used:]])), everything)
