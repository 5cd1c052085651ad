"""Calls on prompts that hold one row in all."""
import pytest
import torch

import prompt_ref as ref
from paper_2411_00853_amd import binding as sv
from paper_2411_00853_amd import workload as wl
from test_gpu_prompt import GROUPED, WIDE, plain_logits, rms, setup

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("hq,hk,hd", [(4, 2, 64), (3, 1, 128), (8, 8, 64)])
@pytest.mark.parametrize("pages", (0, 9))
@pytest.mark.parametrize("apart", (False, True))
def test_append_of_one_row_in_place(hq, hk, hd, pages, apart):
    """As out of place; apart: the row is one of a wider tensor's."""
    h, _, _ = ref.handle(1, hq, hk, hd, 3, 96, pages=pages)
    cols, rot = (hq + 2 * hk) * hd, (hq + hk) * hd
    row0, slot, pos = ref.ints([0, 1]), ref.ints([1]), ref.ints([37])
    place = ref.normal(1, 3, cols + 24, dtype=BF16)[1:2, 8:8 + cols] if apart else ref.normal(1, 1, cols, dtype=BF16)
    before, rotated = place.clone(), torch.empty((1, rot), dtype=BF16, device="cuda")
    caches = []
    for qkv, out in ((before, rotated), (place, place[:, :rot])):
        sv.spec_prompt_append(h, 0, qkv, out, row0, slot, pos)
        kv = torch.empty((1, 2, hk, 1, hd), dtype=BF16, device="cuda")
        sv.spec_kv_export(h, 1, 37, kv)
        caches.append(kv)
    sv.spec_verify_poll(h)
    assert torch.equal(place[:, :rot], rotated) and torch.equal(place[:, rot:], before[:, rot:]) and torch.equal(*caches)
    assert torch.equal(caches[0][0, 0].reshape(1, -1), rotated[:, hq * hd:])


def test_several_rows_in_place_need_one_distance():
    h, _, _ = ref.handle(1, 4, 2, 64, 3, 96)
    x, row0, slot = ref.normal(1, 2, 512, dtype=BF16), ref.ints([0, 2]), ref.ints([0])
    at = [sv._ptr(t) for t in (x, row0, slot)]
    append = lambda rows, ld: sv.lib().spec_prompt_append(h.ptr, 0, at[0], 512, at[0], ld, at[1], at[2], None, 1, rows, None)
    assert append(2, 384) == -1 and b"in place" in sv.lib().spec_last_error()
    assert append(1, 384) == 0 and append(2, 512) == 0
    sv.spec_verify_poll(h)


@pytest.mark.parametrize("shape", (GROUPED, WIDE))
@pytest.mark.parametrize("pages", (0, 6))
def test_a_pass_of_one_token(shape, pages):
    """As near the plain decoder as longer prompts' rows are, and as the same token among others is."""
    w, h, kv_len, prompt = setup(shape, 2, 64, 9, pages)
    tokens = wl.Rng(6, "cuda").randint(0, (9,), shape.vocab)
    slot = ref.ints([1])
    got = prompt.run(tokens[:1].contiguous(), ref.ints([0, 1]), slot).clone()
    sv.spec_verify_poll(h)
    exact, plain = (plain_logits(shape, w, tokens[:1], on)[0] for on in (False, True))
    noise = rms(plain - exact)
    assert rms(got[0] - exact) < 2 * noise and rms(got[0] - plain) < 1.9 * noise
    among = prompt.run(tokens, ref.ints([0, 1, 9]), ref.ints([1, 0]))
    assert rms(among[0] - got[0]) < 0.01 * rms(got[0])


def test_a_context_of_two_tokens():
    from paper_2411_00853_amd.draft8 import Draft8, Rounds
    w, K = wl.make_weights(GROUPED, 5, "cuda", std=0.05), 3
    rounds = Rounds(GROUPED, w, Draft8(GROUPED, w, 1, 64, 16), K, prompt_rows=8)
    rounds.feed(wl.Rng(9, "cuda").randint(0, (1, 2), GROUPED.vocab))
    assert rounds.kv_len.tolist() == [1]
    rounds.propose(torch.full((K, 1), 0.5, device="cuda"))
    rounds.verify(torch.full((1, K + 1), 0.5, device="cuda"), 1.0)
    sv.spec_verify_poll(rounds.handle)
    assert 0 <= int(rounds.n_accepted[0]) <= K
