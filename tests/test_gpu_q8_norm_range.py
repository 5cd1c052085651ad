"""RMSNorm into 8 bits of rows whose squares leave fp32's range."""
import math

import pytest
import torch

import q8_ref as ref
from paper_2411_00853_amd import binding as sv
from test_gpu_q8_rows import SLACK_NORM, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("k", [1, 64, 130, 2048, 4096, 9000, 20000, 65536])
def test_large_rows(k, dtype):
    x = rows(k, 5, k, dtype).clamp_(-64, 64)
    for i, size in enumerate((1e18, 1e19, 1e25, 4e36)):     # the last row stays ordinary
        x[i] = (x[i].float() * size).to(x.dtype)
    gain = 1 + 0.3 * torch.randn(k, device="cuda")
    h = torch.empty_like(x)
    q, s = sv.spec_q8_add_rmsnorm(x, None, gain, 1e-5, h)
    assert torch.equal(h, x)
    y = x.double() / torch.sqrt(x.double().square().mean(1, keepdim=True) + 1e-5) * gain.double()
    ref.check_rows(q, s, y, SLACK_NORM)


@pytest.mark.parametrize("k", [1, 64, 2048, 9000])
def test_small_rows_without_an_epsilon(k):
    x = rows(k + 1, 4, k, "fp32").clamp_(-64, 64)
    x[x.abs() < 1e-3] = 1e-3
    for i, size in enumerate((1e-15, 1e-20, 1e-30, 1e-36)):
        x[i] *= size
    gain = 1 + 0.3 * torch.randn(k, device="cuda")
    q, s = sv.spec_q8_add_rmsnorm(x, None, gain, 0.0)
    y = x.double() / torch.sqrt(x.double().square().mean(1, keepdim=True)) * gain.double()
    ref.check_rows(q, s, y, SLACK_NORM)


@pytest.mark.parametrize("k", [64, 4096, 20000])
def test_infinities_and_nans_keep_their_rows(k):
    """A NaN anywhere makes the row NaN; an infinity its block, and zeros of the rest."""
    x = torch.ones((3, k), device="cuda") * 1e25
    x[0, k // 2], x[1, k // 2] = math.nan, math.inf
    q, s = sv.spec_q8_add_rmsnorm(x, None, torch.ones(k, device="cuda"), 1e-5)
    v = (q.float().view(3, -1, 128) * s.t()[..., None]).reshape(3, -1)[:, :k]
    assert bool(v[0].isnan().all())
    blk = k // 2 // 128
    inside = torch.arange(k, device="cuda") // 128 == blk
    assert bool(v[1][inside].isnan().all()) and bool((v[1][~inside] == 0).all())
    assert torch.all((v[2] - 1).abs() <= 2.0 ** -4)
