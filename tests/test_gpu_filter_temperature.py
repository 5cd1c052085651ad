"""Filtered draws at temperatures whose reciprocal is no fp32 number, and at the other end of fp32's range."""
import math

import pytest
import torch

from paper_2411_00853_amd import binding as sv

pytestmark = pytest.mark.gpu

FILTERS = {"": (None, None, None), "k": (2, None, None), "p": (None, 0.5, None), "m": (None, None, 0.3), "kpm": (3, 0.9, 0.5), "k2000": (2000, 0.99, None)}
# of three equal largest logits: top-k of two keeps two, half the mass of three is reached by the second, 0.9 of it by the third
KEPT = {"": 3, "k": 2, "p": 2, "m": 3, "kpm": 3, "k2000": 3}


def draw(x, u, t, filters, workspace):
    rows, vocab = x.shape
    full = lambda v, dtype: None if v is None else torch.full((rows,), v, dtype=dtype, device="cuda")  # noqa: E731
    k, p, mp = filters
    tokens, kept = (torch.full((rows,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    lp, out = torch.full((rows,), 9.0, device="cuda"), torch.full((rows, vocab), 5.0, device="cuda")
    nb = sv.spec_filter_workspace_bytes(rows, vocab) if workspace else 0
    ws = torch.full((nb // 4,), -1, dtype=torch.int32, device="cuda") if nb else None
    sv.spec_filter_sample(x, u, full(t, torch.float32), tokens, full(k, torch.int32), full(p, torch.float32), full(mp, torch.float32), lp, kept, out, ws)
    return tokens, kept, lp, out


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("on", list(FILTERS))
@pytest.mark.parametrize("vocab", [3, 1000, 20000, 70001])
@pytest.mark.parametrize("t", [2.0 ** -126, 2.0 ** -127, 2.0 ** -128, 1e-39, 1e-40, 2.0 ** -149])
def test_smallest_temperatures_leave_the_largest_logits(t, vocab, on, dtype, workspace):
    """Any difference of two logits is many times such a temperature: what is as large as the largest has all the mass."""
    print(t, vocab, on, dtype, workspace, flush=True)
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.randn((4, vocab), generator=g, device="cuda").to(dtype)
    ids = sorted({vocab // 7, vocab // 2, vocab - 1}) if vocab > 3 else [0, 1, 2]
    x[:, ids] = 20.0
    u = torch.tensor([0.0, 0.4, 0.6, 0.999], device="cuda")
    tokens, kept, lp, out = draw(x, u, t, FILTERS[on], workspace)
    n = KEPT[on]
    assert kept.tolist() == [n] * 4
    assert tokens.tolist() == [ids[int(v * n)] for v in (0.0, 0.4, 0.6, 0.999)]
    assert torch.all((lp + math.log(n)).abs() <= 2.0 ** -22)      # one rounding to fp32 of a number below 2
    want = torch.full((4, vocab), -math.inf, device="cuda")
    want[:, ids[:n]] = 20.0
    assert torch.equal(out, want)


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("on", list(FILTERS))
@pytest.mark.parametrize("t", [3.4028234e38, math.inf])
def test_largest_temperatures_make_all_equal(t, on, workspace):
    vocab = 30000
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((4, vocab), generator=g, device="cuda")
    u = torch.tensor([0.0, 0.4, 0.6, 0.999], device="cuda")
    tokens, kept, lp, out = draw(x, u, t, FILTERS[on], workspace)
    k, p, mp = FILTERS[on]
    n = k or vocab
    n = math.ceil(float(torch.tensor(p)) * n) if p else n         # fp32's p of n equal masses
    assert kept.tolist() == [n] * 4
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :n].sort(-1).values
    assert tokens.tolist() == [int(order[r, int(float(u[r]) * n)]) for r in range(4)]
    assert torch.all((lp + math.log(n)).abs() <= 2.0 ** -20)
    assert torch.equal(out > -math.inf, torch.zeros_like(out, dtype=torch.bool).scatter_(1, order, True))
