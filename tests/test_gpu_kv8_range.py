"""Attention over the 8-bit cache at the ends of fp32's range."""
import pytest
import torch

from test_gpu_kv8 import Setup, check_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("size", [1e20, 1e24])
@pytest.mark.parametrize("lens,win,hq,hk,hd", [([0, 40], [1, 3], 4, 2, 64), ([700, 5], [2, 6], 8, 1, 128), ([3000], [1], 8, 8, 128)])
def test_scores_that_are_all_far_below_zero(lens, win, hq, hk, hd, size, workspace):
    """Scores around -10^33 and -10^37: the largest of them has all the weight (the next one is further away than any exponential reaches, and
    than fp32 rounds)."""
    st = Setup(31, lens, win, hq, hk, hd, spread=0.0)
    st.data.view(torch.uint8)[:, :, 0] |= 0x80          # all keys are negative
    st.scales[:, :, 0] = 2.0 ** 30
    q = (st.randn(sum(win), hq * hd).abs() * size).to(torch.bfloat16)
    out = check_attention(st, workspace, scale=1.0, q=q)
    assert not bool((out == 0).all(-1).any())
