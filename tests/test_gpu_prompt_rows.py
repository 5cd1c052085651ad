"""RMSNorm to bf16 and the rotary embedding with the cache's new entries."""
import pytest
import torch

import prompt_ref as ref
from paper_2411_00853_amd import binding as sv

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 64), (1, 512), (6, 513), (9, 1000), (3, 1024), (2, 1025), (7, 2048), (4, 2050), (5, 4096), (3, 5504),
                                       (2, 8192), (2, 11008), (2, 20000), (1, 65536)])
@pytest.mark.parametrize("dtype", (F32, BF16))
def test_norm(rows, cols, dtype):
    """The sum of squares: at most cols 2^-24 of it, half of that in the root; a handful of roundings; one to bf16."""
    x, gain = ref.normal(1, rows, cols, std=3.0, dtype=dtype), 1 + ref.normal(2, cols, std=0.2)
    want = x.double() * torch.rsqrt(x.double().square().mean(-1, keepdim=True) + 1e-5) * gain.double()
    y = sv.spec_prompt_rmsnorm(x, gain, 1e-5)
    assert y.dtype == BF16 and torch.all((y.double() - want).abs() <= want.abs() * (ref.HALF_BF16 + (cols / 2 + 8) * 2.0 ** -24) + 1e-38)


def test_norm_strides_and_neighbours():
    wide = torch.full((5, 200), float("nan"), device="cuda")
    wide[:, 33:133] = ref.normal(1, 5, 100)
    big = torch.full((7, 100), 7.0, dtype=BF16, device="cuda")
    sv.spec_prompt_rmsnorm(wide[:, 33:133], torch.ones(100, device="cuda"), 1e-5, big[1:6])
    x = wide[:, 33:133].double()
    want = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5)
    assert torch.all((big[1:6].double() - want).abs() <= want.abs() * ref.HALF_BF16 * 1.01)
    assert torch.all(big[0] == 7) and torch.all(big[6] == 7)


@pytest.mark.parametrize("cols", (64, 600, 2048, 6000, 20000))
def test_norm_of_rows_whose_squares_leave_fp32(cols):
    x = ref.normal(1, 6, cols)
    x[0] *= 1e30
    x[1] *= 1e-30
    x[3] = 0.0
    x[4, 5 % cols] = float("inf")
    x[5, 5 % cols] = float("nan")
    y = sv.spec_prompt_rmsnorm(x, torch.ones(cols, device="cuda"), 0.0).double()
    want = x[:3].double() * torch.rsqrt(x[:3].double().square().mean(-1, keepdim=True))
    assert torch.all((y[:3] - want).abs() <= want.abs() * (ref.HALF_BF16 + cols * 2.0 ** -24) + 1e-38)
    assert torch.isnan(y[5]).all() and torch.isnan(y[4, 5]) and torch.all((y[4].nan_to_num(0) == 0))
    assert torch.all(sv.spec_prompt_rmsnorm(x[3:4], torch.ones(cols, device="cuda"), 1e-5) == 0)


# ---- append -------------------------------------------------------------------------------------------

def check_append(h, cache_of, qkv, rotated, lens, pos, slots, layer, before=None):
    """cache_of(slot, pos0, n) -> [2][kv heads][n][hd] of the layer"""
    c = h.cfg
    hq, hk, hd = c.n_q_heads, c.n_kv_heads, c.head_dim
    row = 0
    for n, p, s in zip(lens, pos, slots):
        x = qkv[row:row + n].double().reshape(n, hq + 2 * hk, hd)
        want = ref.rotate(x[:, :hq + hk], p + torch.arange(n, device="cuda"), c.rope_theta)
        got = rotated[row:row + n].double().reshape(n, hq + hk, hd)
        size = x[:, :hq + hk].abs()
        size = size + size.roll(hd // 2, -1)
        assert torch.all((got - want).abs() <= want.abs() * ref.HALF_BF16 + size * 2.0 ** -22)
        if n:
            kv = cache_of(s, p, n)
            assert torch.equal(kv[0], rotated[row:row + n].reshape(n, hq + hk, hd)[:, hq:].transpose(0, 1))
            assert torch.equal(kv[1], qkv[row:row + n].reshape(n, hq + 2 * hk, hd)[:, hq + hk:].transpose(0, 1))
        row += n


def exporter(h, layer):
    def get(slot, pos0, n):
        c = h.cfg
        out = torch.empty((c.n_layers, 2, c.n_kv_heads, n, c.head_dim), dtype=BF16, device="cuda")
        sv.spec_kv_export(h, slot, pos0, out)
        return out[layer]
    return get


@pytest.mark.parametrize("hq,hk,hd", [(4, 2, 64), (3, 1, 128), (8, 8, 64), (32, 32, 128), (6, 2, 128), (12, 4, 64)])
@pytest.mark.parametrize("paged", (False, True))
def test_append(hq, hk, hd, paged):
    slots, max_kv, layers = 4, 200, 2
    h, cache, kv_len = ref.handle(layers, hq, hk, hd, slots, max_kv, pages=slots * 7 if paged else 0)
    lens, pos, where = [1, 70, 0, 33], [0, 31, 5, 100], [2, 0, 3, 1]
    rows = sum(lens)
    row0, seq, pos0 = ref.ints(ref.starts(lens)), ref.ints(where), ref.ints(pos)
    older = ref.normal(9, layers, 2, hk, 31, hd, dtype=BF16)
    sv.spec_kv_import(h, 0, 0, older)
    for layer in range(layers):
        qkv = ref.normal(layer, rows + 2, (hq + 2 * hk) * hd, dtype=BF16)      # (two rows of no sequence behind)
        rotated = torch.full((rows + 2, (hq + hk) * hd), 7.0, dtype=BF16, device="cuda")
        sv.spec_prompt_append(h, layer, qkv, rotated, row0, seq, pos0)
        check_append(h, exporter(h, layer), qkv, rotated, lens, pos, where, layer)
        assert torch.all(rotated[rows:] == 7)
        place = qkv.clone()
        sv.spec_prompt_append(h, layer, place, place[:, :(hq + hk) * hd], row0, seq, pos0)
        assert torch.equal(place[:rows, :(hq + hk) * hd], rotated[:rows]) and torch.equal(place[:, (hq + hk) * hd:], qkv[:, (hq + hk) * hd:])
        assert torch.equal(place[rows:], qkv[rows:])
    sv.spec_verify_poll(h)
    out = torch.empty_like(older)
    sv.spec_kv_export(h, 0, 0, out)
    assert torch.equal(out, older)
    assert torch.all(kv_len == 0)


def test_nothing_but_the_new_positions_changes():
    h, cache, _ = ref.handle(2, 4, 2, 64, 3, 128)
    filled = ref.normal(3, 2, 2, 2, 128, 64, dtype=BF16)
    for s in range(3):
        sv.spec_kv_import(h, s, 0, filled)
    qkv = ref.normal(4, 50, 8 * 64, dtype=BF16)
    rotated = torch.empty((50, 6 * 64), dtype=BF16, device="cuda")
    sv.spec_prompt_append(h, 1, qkv, rotated, ref.ints([0, 50]), ref.ints([1]), ref.ints([41]))
    for s in range(3):
        out = torch.empty_like(filled)
        sv.spec_kv_export(h, s, 0, out)
        if s == 1:
            assert torch.equal(out[1, 1, :, 41:91], qkv.reshape(50, 8, 64)[:, 6:].transpose(0, 1))
            out[1, :, :, 41:91] = filled[1, :, :, 41:91]
        assert torch.equal(out, filled)


def test_one_slot_twice():
    for pages in (0, 12):
        h, _, _ = ref.handle(1, 4, 2, 64, 3, 96, pages=pages)
        lens, pos = [40, 20], [40, 10]
        qkv = ref.normal(4, 60, 8 * 64, dtype=BF16)
        rotated = torch.empty((60, 6 * 64), dtype=BF16, device="cuda")
        sv.spec_prompt_append(h, 0, qkv, rotated, ref.ints([0, 40, 60]), ref.ints([1, 1]), ref.ints(pos))
        sv.spec_verify_poll(h)
        check_append(h, exporter(h, 0), qkv, rotated, lens, pos, [1, 1], 0)
        if pages:
            assert sv.spec_kv_pages(h) == (12 - 3, 12)


@pytest.mark.parametrize("slot,pos,status", [(-1, 0, -1), (3, 0, -1), (1, -1, -3), (1, 70, -3), (1, 2 ** 31 - 5, -3)])
@pytest.mark.parametrize("pages", (0, 9))
def test_sequences_that_do_not_fit_are_skipped(slot, pos, status, pages):
    h, cache, _ = ref.handle(1, 4, 2, 64, 3, 96, pages=pages)
    lens, where, at = [20, 30, 10], [0, slot, 2], [3, pos, 0]
    qkv = ref.normal(4, 60, 8 * 64, dtype=BF16)
    rotated = torch.full((60, 6 * 64), 7.0, dtype=BF16, device="cuda")
    sv.spec_prompt_append(h, 0, qkv, rotated, ref.ints([0, 20, 50, 60]), ref.ints(where), ref.ints(at))
    with pytest.raises(sv.SpecError) as e:
        sv.spec_verify_poll(h)
    assert e.value.status == status
    assert torch.all(rotated[20:50] == 0)
    keep = list(range(20)) + list(range(50, 60))
    check_append(h, exporter(h, 0), qkv[keep], rotated[keep], [20, 10], [3, 0], [0, 2], 0)
    if not pages:
        out = exporter(h, 0)(1, 0, 96)
        assert torch.all(out == 0)


def test_a_pool_that_runs_dry():
    h, cache, _ = ref.handle(1, 4, 2, 64, 2, 96, pages=2)
    qkv = ref.normal(4, 90, 8 * 64, dtype=BF16)
    rotated = torch.empty((90, 6 * 64), dtype=BF16, device="cuda")
    sv.spec_prompt_append(h, 0, qkv, rotated, ref.ints([0, 90]), ref.ints([1]))
    with pytest.raises(sv.SpecError) as e:
        sv.spec_verify_poll(h)
    assert e.value.status == -3
    check_append(h, exporter(h, 0), qkv[:64], rotated[:64], [64], [0], [1], 0)
    assert torch.all(rotated[64:].abs().sum(1) > 0)


def test_append_replayed():
    h, _, _ = ref.handle(1, 4, 2, 64, 3, 96, pages=9)
    qkv = ref.normal(4, 40, 8 * 64, dtype=BF16)
    rotated = torch.empty((40, 6 * 64), dtype=BF16, device="cuda")
    row0, seq, pos0 = ref.ints([0, 25, 40]), ref.ints([0, 1]), ref.ints([0, 7])
    sv.spec_prompt_append(h, 0, qkv, rotated, row0, seq, pos0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sv.spec_prompt_append(h, 0, qkv, rotated, row0, seq, pos0)
    for lens, pos, where in (([25, 15], [0, 7], [0, 1]), ([10, 30], [40, 60], [2, 1]), ([0, 40], [0, 50], [2, 2])):
        row0.copy_(ref.ints(ref.starts(lens)))
        pos0.copy_(ref.ints(pos))
        seq.copy_(ref.ints(where))
        qkv.normal_()
        graph.replay()
        torch.cuda.synchronize()
        sv.spec_verify_poll(h)
        check_append(h, exporter(h, 0), qkv, rotated, lens, pos, where, 0)
