"""RMSNorm of rows whose squares, and an eps that, leave fp32's normal numbers."""
import pytest
import torch

import prompt_ref as ref
from paper_2411_00853_amd import binding as sv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", (64, 600, 2048, 6000, 20000))
@pytest.mark.parametrize("eps", (0.0, 1e-44, 1e-42, 1e-40, 1e-38, 1e-33, 1e-30, 1e-20))
def test_small_rows_and_small_eps(cols, eps):
    """The sum of squares: at most cols 2^-24 of it, half of that in the root; the roundings of eps (taken as the float that it is) by powers of two:
    none; a handful of others and one to bf16."""
    sizes = torch.tensor([1.0, 1e30, 1e-15, 1e-18, 1e-19, 1e-20, 1e-21, 1e-22, 1e-23, 1e-30], device="cuda")
    x, gain = ref.normal(1, len(sizes), cols) * sizes[:, None], 1 + ref.normal(2, cols, std=0.2)
    y = sv.spec_prompt_rmsnorm(x, gain, eps).double()
    e = float(torch.tensor(eps, dtype=torch.float32).double())
    want = x.double() * torch.rsqrt(x.double().square().mean(-1, keepdim=True) + e) * gain.double()
    off = ((y - want).abs() - want.abs() * (ref.HALF_BF16 + (cols / 2 + 8) * 2.0 ** -24) - 1e-38).amax(1)
    assert torch.all(off <= 0), off.tolist()
    if eps:
        assert torch.all(sv.spec_prompt_rmsnorm(torch.zeros((3, cols), device="cuda"), gain, eps) == 0)
