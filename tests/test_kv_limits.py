"""Sizes at the ends of what the key/value cache's entry points accept (no GPU needed): what a kernel
could not step through, and what no launch can hold, is refused before anything is launched."""
import pytest

from test_kv_abi import CALLS, Call, kv, refused  # noqa: F401

MOST = 2 ** 31 - 4097  # tokens of a sequence


def long(c, tokens):
    c.seqs.table_stride = c.seqs.table_width = 1 << 27
    c.seqs.longest = tokens
    return c


@pytest.mark.parametrize("tokens", [MOST + 1, 2 ** 31 - 64, 2 ** 31 - 1, 2 ** 31, 2 ** 33])
def test_sequences_too_long_to_step_through(kv, tokens):  # noqa: F811
    c = long(Call(kv), tokens)
    for call in CALLS:
        assert getattr(c, call)() == -1, call
    assert c.size(kv.OP_ATTEND) == 0 and c.size(kv.OP_SELECT) == 0


def test_the_longest_sequences(kv):  # noqa: F811
    c = long(Call(kv), MOST)
    assert c.size(kv.OP_ATTEND) > 0
    c.keep = 4
    assert c.size(kv.OP_SELECT) > 0
