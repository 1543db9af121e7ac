"""What the handles of the blocks for requests hold after a call."""
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
