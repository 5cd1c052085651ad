"""The rotary embedding of more sequences than a wavefront counts at a time, empty ones and ones that do not fit among them."""
import pytest
import torch

import prompt_ref as ref
from paper_2411_00853_amd import binding as sv
from test_gpu_prompt_rows import check_append, exporter

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hk,hd", [(5, 5, 64), (6, 3, 128)])
@pytest.mark.parametrize("pages", (0, 200 * 4))
def test_two_hundred_sequences(hq, hk, hd, pages):
    slots, max_kv = 200, 128
    h, _, _ = ref.handle(1, hq, hk, hd, slots, max_kv, pages=pages)
    lens = [0 if b % 7 == 3 else (b * 37) % 64 + (b % 5 == 0) for b in range(slots)]
    pos = [(b * 13) % 60 for b in range(slots)]
    where = [(b * 77 + 5) % slots for b in range(slots)]
    rows = sum(lens)
    qkv = ref.normal(1, rows + 3, (hq + 2 * hk) * hd, dtype=ref.BF16)
    rotated = torch.full((rows + 3, (hq + hk) * hd), 7.0, dtype=ref.BF16, device="cuda")
    sv.spec_prompt_append(h, 0, qkv, rotated, ref.ints(ref.starts(lens)), ref.ints(where), ref.ints(pos))
    sv.spec_verify_poll(h)
    check_append(h, exporter(h, 0), qkv, rotated, lens, pos, where, 0)
    assert torch.all(rotated[rows:] == 7)
    if pages:
        assert sv.spec_kv_pages(h)[0] == pages - sum((p + n + 31) // 32 for n, p in zip(lens, pos) if n)
    # some that do not fit
    spoilt = [-1 if b in (2, 70) else slots if b == 130 else s for b, s in enumerate(where)]
    far = [max_kv if b in (65, 199) else p for b, p in enumerate(pos)]
    rotated.fill_(7.0)
    sv.spec_prompt_append(h, 0, qkv, rotated, ref.ints(ref.starts(lens)), ref.ints(spoilt), ref.ints(far))
    with pytest.raises(sv.SpecError):
        sv.spec_verify_poll(h)
    s = ref.starts(lens)
    out = {2, 65, 70, 130, 199}
    for b in out:
        assert torch.all(rotated[s[b]:s[b + 1]] == 0)
    keep = [b for b in range(slots) if b not in out]
    at = torch.tensor([r for b in keep for r in range(s[b], s[b + 1])], device="cuda")
    check_append(h, exporter(h, 0), qkv[at], rotated[at], [lens[b] for b in keep], [pos[b] for b in keep], [where[b] for b in keep], 0)
