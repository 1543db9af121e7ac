"""The operators of a serving step together: blocks given and taken back, rotary positions, the
cache in 4 bits written and attended to, eager and recorded, against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

from gpu_util import dev, host, need_gpu
from kv4_defs import RefCache4
from test_gpu_kv4 import near, of_tiles
from test_gpu_pages import Ref
from test_gpu_rotary import reference

pytestmark = pytest.mark.gpu


def inputs(step, n, seed=5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(step.n_seqs, step.hidden, generator=gen, device="cuda").bfloat16() for _ in range(n)]


def options():
    need_gpu()
    from paper_2203_00448_amd import kv, rotary
    return dict(kind=kv.E2M1, paged=True, rotation=rotary.Rotation(48, scaling="linear", factor=2.0))


def test_planned_step_is_the_same():
    from paper_2203_00448_amd.decode_step import DecodeStep
    opts = options()
    planned, apart = DecodeStep(**opts), DecodeStep(planned=False, **opts)
    assert planned.bytes < planned.unplanned_bytes / 2
    for i, x in enumerate(inputs(planned, 100)):
        assert torch.equal(planned.run(x), apart.run(x))
        if i in (40, 41, 77):
            done = torch.arange(8, device="cuda") % 3 == i % 3
            planned.retire(done)
            apart.retire(done)
    planned.check()
    apart.check()
    assert all(torch.equal(x, y) for a, b in zip(planned.caches, apart.caches) for x, y in zip(a.tensors, b.tensors))
    assert torch.equal(planned.pool.ids, apart.pool.ids)


def test_selection_with_rotation():
    """The 8-bit step's own options: positions without a pool are those with one."""
    from paper_2203_00448_amd import kv
    from paper_2203_00448_amd.decode_step import DecodeStep
    opts = options() | dict(kind=kv.INT8, keep=5)
    a, b = DecodeStep(**opts), DecodeStep(**(opts | dict(paged=False)))
    for x in inputs(a, 120):
        assert torch.equal(a.run(x), b.run(x))
    a.check()
    b.check()


def test_recorded_step():
    from paper_2203_00448_amd.decode_step import DecodeStep
    opts = options()
    eager, recorded = DecodeStep(**opts), DecodeStep(**opts)
    steps = inputs(eager, 60)
    x = steps[0].clone()
    recorded.run(x)  # as a program warms up; forgotten below
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = recorded.run(x)
    recorded.retire(torch.ones(8, dtype=torch.bool, device="cuda"))
    recorded.table.fill_(-1)
    recorded.pool.ids.copy_(eager.pool.ids)
    for i, s in enumerate(steps):
        x.copy_(s)
        graph.replay()
        want = eager.run(s)
        assert torch.equal(out, want), i
        if i % 25 == 24:
            done = torch.arange(8, device="cuda") < 3
            recorded.retire(done)
            eager.retire(done)
    eager.check()
    recorded.check()


def test_against_the_definition():
    """One layer: rows, rotary positions, cache and attention from the step's own projections, in 64 bits.
    The hidden state adds two roundings of a product in bfloat16."""
    from paper_2203_00448_amd.decode_step import DecodeStep
    step = DecodeStep(layers=1, n_seqs=3, longest=256, **options())
    cache, r = step.caches[0], step.rotation
    ref = RefCache4(cache.n_blocks, step.heads, step.dim, cache.block)
    q0, q1 = step.q_heads, step.q_heads + step.heads
    worst = 0.0
    for t, x in enumerate(inputs(step, 100)):
        out = step.run(x).clone()
        # the projected rows as the step rounded them: their memory is done with, so computed again
        rows = torch.mm(x, step.w_in[0]).view(3, -1, step.dim)
        v = host(rows[:, q1:].double())
        turned = reference(host(rows[:, :q1].double()), np.full(3, t), host(r.freq), r.magnitude, r.turned, r.pairs, False)[0]
        turned = host(torch.from_numpy(turned).to(torch.bfloat16).double())
        table = host(step.table).astype(np.int64)
        length, begin = [t + 1] * 3, np.arange(4)
        ref.write(table, length, begin, turned[:, q0:], v)
        result = ref.attend(table, length, begin, turned[:, :q0], step.dim ** -0.5)[0]
        want = host(x.double()) + result.reshape(3, -1) @ host(step.w_out[0].double())
        worst = max(worst, float(np.linalg.norm(host(out.double()) - want) / np.linalg.norm(want)))
    step.check()
    # attention's result, the product and the sum are rounded to 8 bits each: 2^-9 apiece in the mean.  (A turned
    # key that lies between two bfloat16 values may be rounded the other way and then take another code: half a
    # step of 4 bits in one of thousands of values, less than the roundings.)
    assert worst < 3 * 2.0 ** -8


@pytest.mark.parametrize("dtype,dim,block,group", [(torch.bfloat16, 128, 16, 4), (torch.float16, 64, 64, 2)])
def test_requests_come_and_go(dtype, dim, block, group):
    """Prompts of every length beside conversations that go on, in one ragged call each turn: requests end,
    their blocks go to others, what is stored and attended to is each request's own."""
    binding = need_gpu()
    from paper_2203_00448_amd import kv, pages, rotary
    rng = np.random.default_rng(dim)
    n, heads, width = 7, 2, 40
    n_blocks = 7 * 700 // block
    cache = kv.new_cache(n_blocks, heads, dim, block=block, kind=kv.E2M1)
    ids = rng.permutation(n_blocks)
    pool = pages.Pool(dev(ids, torch.int32), torch.zeros(1, dtype=torch.int64, device="cuda"))
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    length = torch.zeros(n, dtype=torch.int32, device="cuda")
    ref = RefCache4(n_blocks, heads, dim, block)
    plan = Ref(ids, 0, np.full((n, width), -1, np.int64), [0] * n, block)
    rotation = rotary.Rotation(dim, pairs=True)
    status = kv.new_status()
    for turn in range(6):
        done = (rng.random(n) < 0.3) & (turn > 0)
        pages.release(pool, table, length, dev(done, torch.bool), block=block, status=status)
        plan.release(done)
        more = [int(rng.integers(1, 150)) if m == 0 else int(rng.integers(0, 3)) for m in plan.length]
        step = pages.new_step(n, sum(more))
        pages.extend(pool, table, length, dev(np.array(more), torch.int32), block=block, step=step, status=status)
        begin, position, slot = plan.extend(more)
        assert list(host(step.slot)) == slot and list(host(step.position)) == position
        rows = torch.from_numpy(rng.standard_normal((sum(more), heads * (group + 2), dim))).to(dtype).cuda()
        q, k, v = rows.split([heads * group, heads, heads], 1)
        rotary.rotate(rotation, step.position, q, k, out=q, k_out=k)
        seqs = kv.Seqs(table, length, begin=step.begin, tokens=sum(more))
        kv.write(cache, seqs, k, v, status=status)
        got = kv.attend(cache, seqs, q, status=status)
        ref.write(plan.table, plan.length, begin, host(k.double()), host(v.double()))
        for name in ("k_code", "v_code", "k_exp", "v_exp"):
            assert np.array_equal(host(getattr(cache, name)), getattr(ref, name)), (turn, name)
        want = ref.attend(plan.table, plan.length, begin, host(q.double()), dim ** -0.5)
        near(got, None, want, dtype, of_tiles(dtype))
        # the slots say where the rows went
        flat = cache.k_code.transpose(1, 2).reshape(-1, heads, dim // 2)[step.slot]
        assert torch.equal(flat, dev(np.stack([ref.k_code[s // block, :, s % block] for s in slot]), torch.uint8))
    assert int(status.item()) == binding.MP_OK


def test_command():
    need_gpu()
    from paper_2203_00448_amd.decode_step import main
    assert main(40)
