"""Blocks given to requests and taken back, on the GPU against plain loops."""
import numpy as np
import pytest
import torch

from gpu_util import dev, host, need_gpu

pytestmark = pytest.mark.gpu


def modules():
    need_gpu()
    from paper_2203_00448_amd import binding, pages
    return binding, pages


class Ref:
    """A pool and a table as a program without a GPU would keep them."""

    def __init__(self, ids, used, table, length, block):
        self.ids, self.used, self.table, self.length, self.block = list(ids), used, table.copy(), list(length), block

    def blocks(self, n):
        return (n + self.block - 1) // self.block

    def release(self, done):
        back = [self.table[s, b] for s in range(len(self.length)) if done[s] for b in range(self.blocks(self.length[s]))]
        self.used -= len(back)
        self.ids[self.used:self.used + len(back)] = back
        self.length = [0 if d else n for d, n in zip(done, self.length)]

    def extend(self, more):
        begin, position, slot = [0], [], []
        for s, m in enumerate(more):
            n = self.length[s]
            for b in range(self.blocks(n), self.blocks(n + m)):
                self.table[s, b] = self.ids[self.used]
                self.used += 1
            position += range(n, n + m)
            slot += [int(self.table[s, p // self.block]) * self.block + p % self.block for p in range(n, n + m)]
            self.length[s] = n + m
            begin.append(begin[-1] + m)
        return begin, position, slot


class Setup:
    def __init__(self, length, *, block=64, width=None, spare=200, seed=0, pad=0):
        self.binding, self.pages = modules()
        rng = np.random.default_rng([seed, block, len(length)])
        need = [(n + block - 1) // block for n in length]
        width = width or max(need + [1]) + 3
        ids = rng.permutation(sum(need) + spare) + 1000
        table = np.full((len(length), width), -5, np.int64)
        at = 0
        for s, n in enumerate(need):
            table[s, :n] = ids[at:at + n]
            at += n
        self.ref = Ref(ids, at, table, length, block)
        self.block, self.n = block, len(length)
        self.pool = self.pages.Pool(dev(ids, torch.int32), dev(np.array([at]), torch.int64))
        room = torch.full((max(1, len(length)), width + pad), -5, dtype=torch.int32, device="cuda")[:len(length)]
        self.table = room[:, :width]
        self.table.copy_(dev(table, torch.int32))
        self.room, self.width = room, width
        self.length = dev(np.array(length), torch.int32)
        self.status = self.binding.new_status()

    def extend(self, more, room=None, **kw):
        total = sum(more) if room is None else room
        step = self.pages.new_step(self.n, total)
        step.position.fill_(-7)
        step.slot.fill_(-7)
        self.pages.extend(self.pool, self.table, self.length, dev(np.array(more), torch.int32), block=self.block,
                          step=step, **kw)
        return step

    def release(self, done, dtype=torch.bool, **kw):
        return self.pages.release(self.pool, self.table, self.length, dev(np.array(done), torch.int32).to(dtype),
                                  block=self.block, **kw)

    def same(self):
        assert int(self.pool.used.item()) == self.ref.used
        assert np.array_equal(host(self.pool.ids), self.ref.ids)
        assert np.array_equal(host(self.table), self.ref.table)
        assert list(host(self.length)) == self.ref.length
        assert bool((self.room[:, self.width:] == -5).all())

    def same_step(self, step, want, room=0):
        begin, position, slot = want
        assert list(host(step.begin)) == begin
        assert list(host(step.position)) == position + [-7] * room
        assert list(host(step.slot)) == slot + [-7] * room


@pytest.mark.parametrize("block", [16, 32, 64])
@pytest.mark.parametrize("length,more", [
    ([0], [1]), ([0], [0]), ([64], [1]), ([63], [1]), ([100, 0, 64, 65], [1, 1, 1, 1]), ([5], [1000]),
    ([0, 0, 0], [0, 700, 0]), ([1, 2, 3, 4, 5], [0, 0, 0, 0, 0]), ([16, 32, 64, 128], [48, 1, 0, 300])])
def test_extend(block, length, more):
    s = Setup(length, block=block, width=70, pad=5)  # 1005 tokens are 63 blocks of 16
    step = s.extend(more)
    s.same_step(step, s.ref.extend(more))
    s.same()


@pytest.mark.parametrize("n,seed", [(1, 0), (63, 1), (64, 2), (65, 3), (300, 4), (3000, 5), (9000, 6), (20000, 7)])
def test_steps_of_a_server(n, seed):
    """Requests end, others go on by a token, new ones bring prompts of every length."""
    rng = np.random.default_rng(seed)
    s = Setup(list(rng.integers(0, 200, n)), block=16, width=40, spare=n * 30, seed=seed)
    for turn in range(3):
        done = rng.random(n) < 0.2
        s.release(done)
        s.ref.release(done)
        s.same()
        more = np.where(np.array(s.ref.length) > 0, rng.random(n) < 0.9, rng.integers(0, 150, n)).astype(int)
        if turn == 1:
            more[:] = 0
            more[n // 2] = 130
        step = s.extend(list(more), room=int(more.sum()) + 70)
        s.same_step(step, s.ref.extend(list(more)), room=70)
        s.same()


def test_long_rows_of_zeros_between():
    """A few requests with new tokens among thousands without: bounds that repeat."""
    n = 5000
    more = [0] * n
    for at, m in ((0, 3), (700, 1), (701, 1), (702, 200), (4999, 2)):
        more[at] = m
    s = Setup([10] * n, block=32, width=10)
    s.same_step(s.extend(more), s.ref.extend(more))
    s.same()


def test_outputs_of_their_own():
    """length_out and used_out apart: what was given in is left, and a call repeats."""
    s = Setup([100, 3, 64], block=32)
    out, used = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    ws = s.pages.workspace(3)
    for _ in range(2):
        step = s.extend([5, 100, 1], length_out=out, used_out=used, workspace=ws)
    begin, position, slot = s.ref.extend([5, 100, 1])
    assert list(host(out)) == s.ref.length and int(used.item()) == s.ref.used
    assert list(host(s.length)) == [100, 3, 64] and int(s.pool.used.item()) == 4 + 1 + 2
    assert list(host(step.slot)) == slot and np.array_equal(host(s.table), s.ref.table)


@pytest.mark.parametrize("dtype", [torch.bool, torch.uint8])
def test_release_all_and_none(dtype):
    s = Setup([1000, 0, 64, 1], block=16)
    s.release([0, 0, 0, 0], dtype)
    s.same()
    s.release([1, 1, 1, 1], dtype)
    s.ref.release([1, 1, 1, 1])
    s.same()
    assert s.ref.used == 0


def test_no_sequences():
    s = Setup([], block=16, width=3)
    step = s.extend([], room=4)
    assert list(host(step.begin)) == [0] and list(host(step.slot)) == [-7] * 4
    s.release([])
    assert int(s.pool.used.item()) == 0


@pytest.mark.parametrize("n", [3, 9000])
def test_errors_change_nothing(n):
    """Too few blocks, too little room, lengths that the table cannot hold: the status word, and all as it was."""
    from paper_2203_00448_amd import binding
    length = [40] * n
    plus = lambda m: [m] + [0] * (n - 2) + [m]  # noqa: E731
    for more, room, status, change in (
            (plus(640), None, binding.MP_ENOSPC, None), (plus(17), 33, binding.MP_ENOSPC, None),
            (plus(-1), 5, binding.MP_EINVAL, None), (plus(1000), None, binding.MP_EINVAL, None),
            (plus(1), None, binding.MP_EINVAL, ("length", -1)), (plus(1), None, binding.MP_EINVAL, ("length", 10 ** 6)),
            (plus(2 ** 31 - 1), 5, binding.MP_EINVAL, None),
            (plus(1), None, binding.MP_EINVAL, ("used", -1)), (plus(1), None, binding.MP_EINVAL, ("used", 10 ** 9))):
        s = Setup(length, block=16, width=43, spare=70)
        if change:
            (s.length if change[0] == "length" else s.pool.used)[0] = change[1]
        before = [x.clone() for x in (s.pool.ids, s.pool.used, s.table, s.length)]
        step = s.pages.new_step(n, sum(more) if room is None else room)
        step.begin.fill_(9)
        for out in (None, torch.full((n,), 77, dtype=torch.int32, device="cuda")):
            with pytest.raises(binding.PlanError) as e:
                s.pages.extend(s.pool, s.table, s.length, dev(np.array(more), torch.int32), block=16, step=step,
                               length_out=out)
            assert e.value.status == status
            assert all(torch.equal(a, b) for a, b in zip(before, (s.pool.ids, s.pool.used, s.table, s.length)))
            assert out is None or torch.equal(out, s.length)
        assert not bool(step.begin.any())
        if change:
            with pytest.raises(binding.PlanError):
                s.release([1] * n)
            assert all(torch.equal(a, b) for a, b in zip(before, (s.pool.ids, s.pool.used, s.table, s.length)))
    s = Setup(length, block=16)
    s.pool.used.fill_(2)  # fewer than these sequences hold
    with pytest.raises(binding.PlanError):
        s.release([1] * n)
    assert list(host(s.length)) == length
    s = Setup(length, block=16)
    s.table[0, 0] = -1
    with pytest.raises(binding.PlanError):
        s.release([1] * n)


def test_recorded():
    """A release and an extend in one graph, replayed with other requests, eager calls between."""
    binding, pages = modules()
    a, b = (Setup([100, 20, 64, 0, 300], block=32, width=60) for _ in range(2))
    more, done = (torch.zeros(5, dtype=t, device="cuda") for t in (torch.int32, torch.bool))
    step, ws, status = pages.new_step(5, 500), pages.workspace(5), binding.new_status()

    def both(s, step, ws):
        pages.release(s.pool, s.table, s.length, done, block=32, workspace=ws, status=status, check=False)
        pages.extend(s.pool, s.table, s.length, more, block=32, step=step, workspace=ws, status=status, check=False)

    both(a, step, ws)  # as a program warms up: nothing ends, nothing is new
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(a, step, ws)
    other, ws2 = pages.new_step(5, 500), pages.workspace(5)
    rng = np.random.default_rng(3)
    for _ in range(6):
        more.copy_(dev(rng.integers(0, 90, 5), torch.int32))
        done.copy_(dev(rng.random(5) < 0.4, torch.bool))
        graph.replay()
        both(b, other, ws2)
        for x, y in ((a.pool.ids, b.pool.ids), (a.pool.used, b.pool.used), (a.table, b.table), (a.length, b.length),
                     (step.begin, other.begin), (step.slot, other.slot), (step.position, other.position)):
            assert torch.equal(x, y)
    assert int(status.item()) == 0


def test_python_refusals():
    binding, pages = modules()
    s = Setup([5, 6], block=16)
    one = torch.ones(2, dtype=torch.int32, device="cuda")
    step = pages.new_step(2, 2)
    ok = dict(block=16, step=step)
    for bad in ({"block": 48}, {"workspace": torch.empty(24, dtype=torch.uint8, device="cuda")}):
        with pytest.raises(binding.PlanError):
            pages.extend(s.pool, s.table, s.length, one, **{**ok, **bad})
    with pytest.raises(TypeError):
        pages.extend(s.pool, s.table, s.length, one.long(), **ok)
    with pytest.raises(ValueError):
        pages.extend(s.pool, s.table, s.length, one[:1], **ok)
    with pytest.raises(ValueError):
        pages.extend(s.pool, s.table[:1].expand(2, -1), s.length, one, **ok)
    with pytest.raises(ValueError):
        pages.extend(s.pool, s.table.t(), s.length, one, **ok)
    with pytest.raises(ValueError):
        pages.extend(s.pool, s.table, s.length, one, block=16, step=pages.new_step(3, 2))
    with pytest.raises(TypeError):
        pages.release(s.pool, s.table, s.length, one, block=16)
    s.same()
