"""Outputs that the 8-bit calls make themselves belong to the stream they are written on: memory of the current stream's could still be in use by
work that is queued there."""
import pytest
import torch

from paper_2411_00853_amd import binding as sv

pytestmark = pytest.mark.gpu


def stream_of(t):
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not of the allocator's")


def calls():
    x = torch.randn((300, 1000), device="cuda")
    w = torch.zeros((700, 900), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    gain = torch.ones(1000, device="cuda")
    return (lambda **on: sv.spec_q8_quantize(x, **on), lambda **on: sv.spec_q8_add_rmsnorm(x, None, gain, 1e-5, **on),
            lambda **on: sv.spec_q8_swiglu(x, **on), lambda **on: (sv.spec_q8_pack_weight(w, **on),))


@pytest.mark.parametrize("i", range(4))
def test_new_outputs_are_of_the_calls_stream(i):
    call = calls()[i]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    want = call()
    assert all(stream_of(t) == torch.cuda.current_stream().cuda_stream for t in want)
    got = call(stream=side)
    side.synchronize()
    assert all(stream_of(t) == side.cuda_stream for t in got)
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(want, got))
    with torch.cuda.stream(side):       # and with no stream named, of the current one
        assert all(stream_of(t) == side.cuda_stream for t in call())
    side.synchronize()
