"""A decode step that is given its own last output: planned memory and memory of its own agree."""
import pytest
import torch

from gpu_util import need_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layers", [1, 2, 4])
def test_output_fed_back(layers):
    need_gpu()
    from paper_2203_00448_amd.decode_step import DecodeStep
    planned, apart = DecodeStep(layers=layers, keep=5), DecodeStep(layers=layers, keep=5, planned=False)
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(planned.n_seqs, planned.hidden, generator=gen, device="cuda").bfloat16()
    a, b = x, x.clone()
    for i in range(60):
        a, b = planned.run(a), apart.run(b)
        assert torch.equal(a, b), i
        for y in (a, b):  # in place, to a size that stays as it was: a step grows it two- or threefold
            y.copy_(y.float() / y.float().norm(dim=1, keepdim=True) * 22)
    planned.check()
    apart.check()


def test_output_outlives_the_step_s_memory():
    """The last output is in none of the memory that the plan uses again."""
    need_gpu()
    from paper_2203_00448_amd.decode_step import DecodeStep
    step = DecodeStep()
    x = torch.randn(step.n_seqs, step.hidden, device="cuda").bfloat16()
    out = step.run(x)
    kept = out.clone()
    step.slab.fill_(0x7f)
    assert torch.equal(out, kept)
