"""Short prompts in buffers made for long ones: what a run computes, and how it is shared out, depends on its own rows alone."""
import pytest
import torch

import prompt_ref as ref
from paper_2411_00853_amd import binding as sv
from paper_2411_00853_amd import workload as wl
from paper_2411_00853_amd.prompt import Prompt
from test_gpu_prompt import setup

pytestmark = pytest.mark.gpu
SHAPE = wl.ModelShape(1, 1024, 4, 1, 128, 4096, 1000)       # its products of few rows are shared out, and one prompt's keys


@pytest.mark.parametrize("lens", ([1], [37], [100], [30, 70, 1], [900], [1500]))
def test_a_run_is_the_same_in_larger_buffers(lens):
    rows = sum(lens)
    _, h, _, large = setup(SHAPE, 3, 1536, 4096)
    own = Prompt(h, large.weights, rows, len(lens))
    tokens = wl.Rng(7, "cuda").randint(0, (rows,), SHAPE.vocab)
    where = ref.ints(ref.starts(lens)), ref.ints(list(range(len(lens))))
    want = own.run(tokens, *where, max(lens)).clone()
    large.work.fill_(255)       # (NaN wherever a float is read that was not written)
    assert torch.equal(large.run(tokens, *where, max(lens)), want)
    sv.spec_verify_poll(h)


def test_the_shape_is_shared_out():
    assert sv.spec_prompt_gemm_workspace_bytes(37, 1024, 4096) > 0 and sv.spec_prompt_gemm_workspace_bytes(4096, 1024, 4096) == 0
