"""One batch's handle used by several threads, for caches of different blocks (no GPU needed: the
queries of workspace sizes, on tensors in host memory)."""
import sys
import threading

import pytest
import torch


@pytest.fixture
def kv(monkeypatch):
    from paper_2203_00448_amd import kv
    kv.load_library()
    monkeypatch.setattr(kv, "_need", lambda *a: None)  # host tensors are refused otherwise
    return kv


def test_sequences_shared_by_threads(kv):
    seqs = kv.Seqs(torch.zeros(3, 1000, dtype=torch.int32), torch.zeros(3, dtype=torch.int32))
    caches = [kv.new_cache(4, 2, 64, block=b, device="cpu") for b in (16, 32, 64)]
    want = [kv.workspace_size(kv.OP_ATTEND, c, seqs, q_heads=8) for c in caches]
    assert len(set(want)) > 1 and 0 not in want
    wrong = []

    def ask(i):
        for _ in range(4000):
            got = kv.workspace_size(kv.OP_ATTEND, caches[i], seqs, q_heads=8)
            if got != want[i]:
                wrong.append((i, got))

    was = sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    try:
        threads = [threading.Thread(target=ask, args=(i,)) for i in range(3)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(was)
    assert not wrong, (len(wrong), wrong[:3])


def test_a_bound_that_changes_is_seen(kv):
    seqs = kv.Seqs(torch.zeros(3, 1000, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), longest=5000)
    cache = kv.new_cache(4, 2, 64, block=16, device="cpu")
    sizes = []
    for seqs.longest in (5000, 16000, 5000):
        sizes.append(kv.workspace_size(kv.OP_ATTEND, cache, seqs, q_heads=8))
    assert sizes[0] == sizes[2] != sizes[1]
