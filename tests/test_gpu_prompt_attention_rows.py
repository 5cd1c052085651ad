"""A row of the attention has the same bits whatever the other rows' numbers are: those of its tile too, whose maxima rise at other blocks than its own."""
import pytest
import torch

import prompt_ref as ref
from paper_2411_00853_amd import binding as sv

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def run(q, k, v, hq, hk, n, m, ws):
    out = torch.full_like(q, 7.0)
    sv.spec_prompt_attention(q, k, v, hq, hk, ref.ints([0, n]), out, (q.shape[1] // hq) ** -0.5, k_row0=ref.ints([0, m]), max_q_len=n, max_k_len=m, workspace=ws)
    return out


@pytest.mark.parametrize("n,m", [(900, 900), (40, 1200), (3, 4000), (1, 2000), (12, 3000)])
@pytest.mark.parametrize("hq,hk,hd", [(2, 2, 64), (1, 1, 128), (4, 1, 64), (12, 2, 128)])
@pytest.mark.parametrize("with_work", (False, True))
def test_other_rows_numbers_do_not_matter(n, m, hq, hk, hd, with_work):
    q, k, v = ref.normal(1, n, hq * hd, dtype=BF16), ref.normal(2, m, hk * hd, dtype=BF16), ref.normal(3, m, hk * hd, dtype=BF16)
    size = sv.spec_prompt_attention_workspace_bytes(n, 1, hq, hk, hd) if with_work else 0
    ws = torch.full((max(16, size),), 255, dtype=torch.uint8, device="cuda")
    other = q.reshape(n * hq, hd).clone()      # a row of the kernel is one head of one position
    other[1::2] *= 20
    other[1::4] *= -1
    a, b = (run(t.reshape(n, hq * hd), k, v, hq, hk, n, m, ws).reshape(n * hq, hd) for t in (q, other))
    assert torch.equal(a[::2], b[::2])
    if n * hq > 1:
        assert not torch.equal(a[1::2], b[1::2])
