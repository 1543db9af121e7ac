"""Lists of blocks for rows that see nothing: any block named there is past the row's position."""
import pytest
import torch

from test_gpu_kv import Setup, raised

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block", [16, 64])
def test_blocks_named_for_rows_that_see_nothing(block):
    s = Setup([3, 100], block=block, garbage=False)
    s.fill()
    # five rows of a sequence of three tokens: two that see nothing
    seqs, begin = s.seqs([3, 100], [5, 1])
    q = s.rows(6, 4)
    for named in (-1, 0, 1, -2):
        blocks = torch.full((6, 2, 2), -1, dtype=torch.int32, device="cuda")
        blocks[2:, :, 0] = 0
        blocks[1, 1, 1] = named
        out = torch.full_like(q, 3.0)
        got = raised(s, lambda st: s.kv.attend(s.cache, seqs, q, blocks=blocks, out=out, status=st, check=False))
        assert got == (0 if named == -1 else -1), named
        assert not out[:2].any() and out[2:].any(), named
