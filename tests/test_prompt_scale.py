"""Scales whose logarithm-of-two form leaves fp32 (a score of zero would be no number) are refused (no GPU needed)."""
import ctypes as C

import pytest

from paper_2411_00853_amd import binding as sv

PLACE = 4096      # never dereferenced


@pytest.mark.parametrize("scale,refused", [(2.4e38, True), (-2.4e38, True), (3.4e38, True), (2.3e38, False), (-2.3e38, False), (0.0, False)])
def test_scales(scale, refused):
    a = sv.spec_prompt_attn_args(PLACE, PLACE, PLACE, 512, 128, 128, 512, PLACE, None, 8, 2, 64, 3, 0, 0, 0, 0, scale, PLACE)     # (no rows: nothing is launched)
    rc, message = sv.lib().spec_prompt_attention(C.byref(a), None, 0, None), sv.lib().spec_last_error()
    assert (rc == -1 and b"scale" in message) if refused else rc == 0
