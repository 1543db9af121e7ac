"""A decode step over blocks from a pool whose tokens are refused: what the caches hold stays as it was, and the
steps after it go on."""
import pytest
import torch

from gpu_util import need_gpu

pytestmark = pytest.mark.gpu


def steps(kind, **more):
    binding = need_gpu()
    from paper_2203_00448_amd import kv, rotary
    from paper_2203_00448_amd.decode_step import DecodeStep
    opts = dict(layers=2, n_seqs=3, longest=48, block=16, paged=True, kind=getattr(kv, kind), keep=3,
                rotation=rotary.Rotation(64)) | more
    gen = torch.Generator(device="cuda").manual_seed(3)
    xs = [torch.randn(3, 512, generator=gen, device="cuda").bfloat16() for _ in range(64)]
    return binding, DecodeStep(**opts), DecodeStep(**opts), xs


def held(step):
    return [t.clone() for c in step.caches for t in c.tensors] + [
        step.table.clone(), step.length.clone(), step.pool.ids.clone(), step.pool.used.clone()]


@pytest.mark.parametrize("kind", ["E2M1", "INT8", "E4M3"])
@pytest.mark.parametrize("recorded", [False, True])
def test_a_sequence_at_its_end(kind, recorded):
    """One sequence is as long as it may be, the others are not: a step refuses all of them, and no token of any is
    written over."""
    binding, step, twin, xs = steps(kind)
    done = torch.tensor([False, True, True], device="cuda")
    for i in range(48):
        if i == 20:
            step.retire(done)
            twin.retire(done)
        step.run(xs[i])
        twin.run(xs[i])
    step.check()
    assert step.length.tolist() == [48, 28, 28]
    before = held(step)
    if recorded:
        x = xs[48].clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step.run(x)
        graph.replay()
        graph.replay()
    else:
        step.run(xs[48])
        step.run(xs[49])
    assert all(torch.equal(a, b) for a, b in zip(before, held(step)))
    with pytest.raises(binding.PlanError) as e:
        step.check()
    assert e.value.status == binding.MP_EINVAL
    # the caller lets that sequence go, and the steps are those of a program that had done so in time
    step.status.zero_()
    for s in (step, twin):
        s.retire(~done)
    for x in xs[50:60]:
        assert torch.equal(step.run(x), twin.run(x))
    step.check()
    twin.check()
    assert all(torch.equal(a, b) for a, b in zip(held(step), held(twin)))


def test_a_pool_that_is_short():
    """Fewer blocks than a step needs: refused the same way."""
    binding, step, _, xs = steps("E2M1")
    for x in xs[:16]:
        step.run(x)
    step.check()
    step.pool.used.fill_(step.pool.ids.numel() - 2)  # two free, three sequences at the end of a block
    before = held(step)
    step.run(xs[16])
    assert all(torch.equal(a, b) for a, b in zip(before, held(step)))
    with pytest.raises(binding.PlanError) as e:
        step.check()
    assert e.value.status in (binding.MP_ENOSPC, binding.MP_EINVAL)
