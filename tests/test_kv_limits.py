"""Sizes at the ends of what the key/value cache's entry points accept (no GPU needed): what a kernel
could not step through, and what no launch can hold, is refused before anything is launched."""
import ctypes

import pytest

from test_kv_abi import CALLS, Call, kv  # noqa: F401

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
    c.seqs.n_seqs = c.seqs.n_tokens = 1
    assert c.size(kv.OP_ATTEND) > 0
    c.keep = 4
    assert c.size(kv.OP_SELECT) > 0


def many(kv, sequences, heads, **more):  # noqa: F811
    """A call of one token in all, of the last of so many sequences."""
    c = Call(kv)
    c.cache.heads = c.q_heads = heads
    c.seqs.n_seqs, c.seqs.n_tokens, c.seqs.most_new, c.seqs.longest = sequences, 1, 1, 64
    for name, value in more.items():
        setattr(c.seqs, name, value)
    return c


@pytest.mark.parametrize("sequences,heads,chunks", [(1 << 28, 1 << 16, 1 << 20), (1 << 30, 1 << 16, 1 << 18),
                                                    (1 << 30, 1 << 15, 1 << 19), (1 << 27, 1 << 16, 1 << 20)])
def test_products_past_64_bits(kv, sequences, heads, chunks):  # noqa: F811
    """Row groups times heads times chunks of 2048 tokens would be 2^64 or 2^63."""
    c = many(kv, sequences, heads, table_stride=1 << 27, table_width=1 << 27, longest=chunks * 2048 - 4097)
    assert c.size(kv.OP_ATTEND) == 0
    assert c.attend() == -1


def test_launches_of_too_many_threads(kv):  # noqa: F811
    """2^32 threads or more: 2^24 workgroups of 256, 2^22 of 1024."""
    for call, sequences, heads in (("write", 1 << 21, 4), ("read", 1 << 23, 8), ("attend", 1 << 22, 4),
                                   ("select", 1 << 20, 4)):
        c = many(kv, sequences, heads)
        assert getattr(c, call)() == -1, call
        if call == "attend":
            assert c.size(kv.OP_ATTEND) == 0
    # the join of rows in over 16 chunks: one workgroup a row
    c = Call(kv)
    c.seqs.n_tokens = c.seqs.most_new = 1 << 21
    c.seqs.table_stride = c.seqs.table_width = 1 << 10
    c.seqs.longest = 1 << 16
    c.keep = 1 << 10
    c.blocks = ctypes.c_void_p(1 << 20)
    assert c.size(kv.OP_ATTEND) == 0
    assert c.attend() == -1


def test_launches_that_fit(kv):  # noqa: F811
    c = many(kv, 1 << 20, 4, longest=4096, table_width=64, table_stride=64)
    assert c.size(kv.OP_ATTEND) > 0
    c = many(kv, (1 << 20) - 2, 4, longest=1 << 21, table_width=1 << 15, table_stride=1 << 15)
    assert c.size(kv.OP_SELECT) > 0
