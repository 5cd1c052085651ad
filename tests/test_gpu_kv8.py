"""The 8-bit cache: what an append leaves in its pages, and the attention that reads them, against 64-bit forms."""
import math

import pytest
import torch

import q8_ref as ref
from paper_2411_00853_amd import binding as sv

pytestmark = pytest.mark.gpu


class Setup:
    """A batch of sequences with cached lengths `lens` and windows `win` in a shuffled pool."""

    def __init__(self, seed, lens, win, hq, hk, hd, spread=1.0, max_pos=None):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.win, self.hq, self.hk, self.hd = lens, win, hq, hk, hd
        need = [max(0, -(-(max(n, 0) + w) // 32)) for n, w in zip(lens, win)]
        blocks, pages = max(max(need), 1), sum(need) + 2
        perm = torch.randperm(pages, generator=self.g, device="cuda").to(torch.int32)
        self.table = torch.full((len(lens), blocks), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = perm[at:at + n]
            at += n
        x = self.randn(pages, hk, 2, 32, hd) * torch.exp(spread * self.randn(pages, hk, 2, 1, 1))
        s = ref.pow2_scale(x.double().abs().amax((-1, -2)))
        self.data = ref.make_pages((x / s.float()[..., None, None]).to(ref.F8), hd)
        self.scales = s.float()
        rows = sum(win)
        self.qkv = self.randn(rows, (hq + 2 * hk) * hd).to(torch.bfloat16)
        self.row0 = torch.tensor([0] + torch.tensor(win).cumsum(0).tolist(), dtype=torch.int32, device="cuda")
        self.kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        most = max_pos or max(max(n, 0) + w for n, w in zip(lens, win)) + 1
        ang = torch.arange(most, device="cuda").double()[:, None] * 10000.0 ** (-torch.arange(0, hd, 2, device="cuda").double() / hd)
        self.cos_sin = torch.stack((ang.cos(), ang.sin()), -1).float().contiguous()
        self.max_window = max(win)

    def randn(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda")

    def cache(self):
        return sv.Kv8Cache(self.data, self.scales, self.table, self.hd)

    def held(self, b, n, data=None, scales=None):
        """Positions 0..n-1 of sequence b as fp64 keys and values [n][hk][hd], and which have a page."""
        data, scales = self.data if data is None else data, self.scales if scales is None else scales
        pages = self.table[b, : -(-n // 32)].long()
        ok = (pages >= 0) & (pages < data.shape[0])
        p = pages.clamp(0, data.shape[0] - 1)
        x = ref.page_rows(data.view(torch.uint8)[p].view(ref.F8), self.hd).float().double() * scales[p].double()[..., None, None]
        x = x.permute(2, 0, 3, 1, 4).reshape(2, -1, self.hk, self.hd)[:, :n]
        return x[0], x[1], ok.repeat_interleave(32)[:n]


SLACK = 8 * ref.U    # a rotated key: two products and their sum, each a rounding of a number no larger than the pair's


def check_append(st, rotate=True):
    before, was = st.data.clone(), st.scales.clone()
    q = torch.full((sum(st.win), st.hq * st.hd), 7.0, dtype=torch.bfloat16, device="cuda")
    sv.spec_kv8_append(st.cache(), st.qkv, st.row0, st.kv_len, st.hq, st.max_window, st.cos_sin if rotate else None, q)
    touched = torch.zeros(st.data.shape[0], dtype=torch.bool, device="cuda")
    for b, (n, w) in enumerate(zip(st.lens, st.win)):
        if not w:
            continue
        r0 = int(st.row0[b])
        x = st.qkv[r0:r0 + w].double().reshape(w, st.hq + 2 * st.hk, st.hd)
        rot = ref.rotate(x, st.cos_sin[n:n + w]) if rotate else x
        got = q[r0:r0 + w].double().reshape(w, st.hq, st.hd)
        pair = (x[:, :st.hq, : st.hd // 2].abs() + x[:, :st.hq, st.hd // 2:].abs()).repeat(1, 1, 2)
        assert torch.all((got - rot[:, :st.hq]).abs() <= 2.0 ** -8 * rot[:, :st.hq].abs() + SLACK * pair)
        new = torch.stack((rot[:, st.hq:st.hq + st.hk], x[:, st.hq + st.hk:]), 1)      # [w][2][hk][hd]
        size = torch.stack((x[:, st.hq:st.hq + st.hk], x[:, st.hq + st.hk:]), 1).abs()
        size = size[..., : st.hd // 2] + size[..., st.hd // 2:]
        for blk in range(n // 32, -(-(n + w) // 32)):
            page = int(st.table[b, blk])
            touched[page] = True
            lo, hi = max(32 * blk, n), min(32 * blk + 32, n + w)
            part = new[lo - n:hi - n].permute(1, 2, 0, 3)                              # [2][hk][fresh][hd]
            room = size[lo - n:hi - n].permute(1, 2, 0, 3).repeat(1, 1, 1, 2)
            s = ref.pow2_scale(part.abs().amax((-1, -2))).t()                          # [hk][2]
            if 32 * blk < n:
                s = torch.maximum(s, was[page].double())
            assert torch.equal(st.scales[page].double(), s)
            now = ref.page_rows(st.data[page], st.hd).float().double().permute(1, 0, 2, 3)     # [2][hk][32][hd]
            old = ref.page_rows(before[page], st.hd).float().double().permute(1, 0, 2, 3)
            t = slice(lo - 32 * blk, hi - 32 * blk)
            su = s.t()[..., None, None]
            half = SLACK * room / su
            ok = ref.within_half_step(now[:, :, t], part / su) | ref.within_half_step(now[:, :, t], part / su + half) | \
                ref.within_half_step(now[:, :, t], part / su - half)
            assert bool(ok.all())
            older = old[:, :, : t.start] * (was[page].double().t()[..., None, None] / su) if 32 * blk < n else old[:, :, : t.start]
            assert torch.equal(now[:, :, : t.start], older.float().to(ref.F8).double())
            assert torch.equal(now[:, :, t.stop:], old[:, :, t.stop:])
    assert torch.equal(st.data.view(torch.uint8)[~touched], before.view(torch.uint8)[~touched])
    assert torch.equal(st.scales[~touched], was[~touched])
    return q


APPENDS = [([0], [1], 4, 4, 64), ([31], [2], 4, 2, 128), ([5, 100, 64], [3, 1, 40], 8, 2, 64), ([33, 0, 7], [0, 70, 5], 6, 3, 128),
           ([1000], [16], 8, 8, 128), ([95, 96, 97], [1, 1, 1], 2, 1, 64)]


@pytest.mark.parametrize("rotate", [True, False])
@pytest.mark.parametrize("lens,win,hq,hk,hd", APPENDS)
def test_append(lens, win, hq, hk, hd, rotate):
    check_append(Setup(1, lens, win, hq, hk, hd), rotate)


def test_a_growing_scale_rounds_the_older_positions_again():
    st = Setup(2, [20, 40], [2, 3], 4, 2, 64)
    st.qkv *= 300
    check_append(st)
    small = Setup(3, [20, 40], [2, 3], 4, 2, 64)
    small.qkv *= 2.0 ** -30      # the scales stay, the new positions round to zero
    was = small.scales.clone()
    check_append(small)
    assert torch.equal(was, small.scales)


def test_appending_the_same_window_twice_changes_nothing_more():
    st = Setup(4, [50, 31], [6, 3], 8, 4, 128)
    st.qkv *= 20
    q = torch.empty((9, 8 * 128), dtype=torch.bfloat16, device="cuda")
    call = lambda: sv.spec_kv8_append(st.cache(), st.qkv, st.row0, st.kv_len, 8, st.max_window, st.cos_sin, q)  # noqa: E731
    call()
    once, scales = st.data.clone(), st.scales.clone()
    call()
    assert torch.equal(once.view(torch.uint8), st.data.view(torch.uint8)) and torch.equal(scales, st.scales)


def test_append_of_what_is_no_number_and_of_zeros():
    st = Setup(5, [10, 64], [4, 4], 2, 1, 64)
    x = st.qkv.view(8, 4, 64)
    x[1, 2, 3], x[2, 3, 9], x[3, 3, 1] = math.nan, math.inf, -math.inf
    x[4:, 2:] = 0
    was = st.scales.clone()
    sv.spec_kv8_append(st.cache(), st.qkv, st.row0, st.kv_len, 2, 4)
    k, v, _ = st.held(0, 14)
    assert bool(k[11, 0, 3].isnan()) and bool(v[12, 0, 9].isnan()) and bool(v[13, 0, 1].isnan())
    assert int(k.isnan().sum()) == 1 and int(v.isnan().sum()) == 2
    assert torch.all(st.scales[st.table[0, 0].long()] <= torch.maximum(was[st.table[0, 0].long()], torch.tensor(2.0 ** -5, device="cuda")))
    assert torch.all(st.scales[st.table[1, 2].long()] == 2.0 ** -126)
    k, v, _ = st.held(1, 68)
    assert torch.all(k[64:] == 0) and torch.all(v[64:] == 0)


def test_append_without_a_place():
    """Sequences with a negative length, a missing page, a full table, a rotation table that ends: nothing else is touched."""
    st = Setup(6, [-1, 40, 126, 10], [2, 3, 4, 2], 4, 2, 64)
    st.table = st.table[:, :4].contiguous()
    st.table[1, 1] = 99999
    st.cos_sin = st.cos_sin[:127].contiguous()
    before, was = st.data.clone(), st.scales.clone()
    q = torch.full((11, 4 * 64), 7.0, dtype=torch.bfloat16, device="cuda")
    sv.spec_kv8_append(st.cache(), st.qkv, st.row0, st.kv_len, 4, 4, st.cos_sin, q)
    changed = (before.view(torch.uint8) != st.data.view(torch.uint8)).flatten(1).any(1).nonzero().flatten().tolist()
    assert set(changed) <= {int(st.table[2, 3]), int(st.table[3, 0])}
    # 126 has a rotation, 127 has none, 128 and 129 have no place
    assert torch.all(q[:2] == 0) and torch.all(q[6:9] == 0) and not bool((q[5] == 0).all())
    got = ref.page_rows(st.data[int(st.table[2, 3])], 64).view(torch.uint8)
    old = ref.page_rows(before[int(st.table[2, 3])], 64).view(torch.uint8)
    assert torch.equal(got[:, :, 31], old[:, :, 31]) and not torch.equal(got[:, :, 30], old[:, :, 30])
    unlike = [i for i in range(st.scales.shape[0]) if not torch.equal(was[i], st.scales[i])]
    assert set(unlike) <= set(changed)


# ---- attention ---------------------------------------------------------------------------------------------

# weights round to eleven bits (2^-12), scores are fp32 sums of up to 128 products of a magnitude below 64 (4e-4), the result is bf16
REL, WEIGHTS = 2.0 ** -8, 1e-3


def check_attention(st, workspace=True, max_len=None, scale=None, q=None):
    rows = sum(st.win)
    scale = st.hd ** -0.5 if scale is None else scale
    if q is None:
        q = st.randn(rows, st.hq * st.hd).to(torch.bfloat16)
    out = torch.full((rows, st.hq * st.hd), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((sv.spec_kv8_workspace_bytes(rows, st.hq, st.hd) // 4,), float("nan"), device="cuda") if workspace else None
    sv.spec_kv8_attention(st.cache(), q, st.row0, st.kv_len, st.hq, st.max_window,
                          st.table.shape[1] * 32 if max_len is None else max_len, scale, out, ws)
    cap = st.table.shape[1] * 32
    for b, (n, w) in enumerate(zip(st.lens, st.win)):
        if not w:
            continue
        r0 = int(st.row0[b])
        got = out[r0:r0 + w].double().reshape(w, st.hq, st.hd)
        if n < 0:
            assert torch.all(got == 0)
            continue
        length = min(n + w, cap)
        k, v, ok = st.held(b, length)
        where = ok.nonzero().flatten()
        lims = torch.tensor([int((where <= min(n + j, cap - 1)).sum()) - 1 for j in range(w)], device="cuda")
        qd = q[r0:r0 + w].double().reshape(w, st.hq, st.hd)
        want, mag = ref.attend(qd, k[where], v[where], lims, scale)
        off = (got - want).abs()
        bound = REL * want.abs() + WEIGHTS * mag + 1e-30
        assert torch.all(off <= bound), (b, float((off / bound).max()))
    return out


ATTENDS = [([0], [1], 1, 1, 64), ([0], [1], 4, 4, 128), ([1], [1], 8, 1, 64), ([31], [1], 8, 2, 128), ([32], [1], 2, 2, 64),
           ([1023], [1], 8, 2, 64), ([700, 3, 95, 0], [6, 6, 6, 6], 4, 4, 128), ([130, 40, 64], [3, 0, 7], 12, 4, 128),
           ([500], [16], 8, 1, 64), ([77, 200], [33, 12], 6, 2, 64), ([64, 5], [70, 9], 4, 1, 128), ([2500, 12], [2, 1], 32, 4, 64),
           ([10], [200], 2, 2, 64), ([250], [5], 21, 3, 128)]


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("lens,win,hq,hk,hd", ATTENDS)
def test_attention(lens, win, hq, hk, hd, workspace):
    check_attention(Setup(11, lens, win, hq, hk, hd), workspace)


@pytest.mark.parametrize("max_len", [0, 32, 1 << 20])
def test_the_expected_length_changes_no_result_but_its_rounding(max_len):
    check_attention(Setup(12, [900, 30], [2, 2], 8, 2, 128), True, max_len)


def test_a_long_cache():
    check_attention(Setup(13, [40000], [3], 8, 1, 128))
    check_attention(Setup(14, [33333, 17, 9000], [1, 1, 1], 4, 1, 64))


def test_scores_far_apart_and_scales_far_apart():
    st = Setup(15, [600, 90], [4, 4], 4, 2, 128, spread=6.0)      # pages whose scales differ by many powers of two
    check_attention(st)
    st = Setup(16, [600, 90], [4, 4], 4, 2, 64)
    q = (st.randn(8, 4 * 64) * 6).to(torch.bfloat16)              # scores of +-50: one position takes all
    check_attention(st, q=q, scale=1.0)
    st.scales[::3, :, 1] = 2.0 ** -126                            # pages of values that count as nothing
    st.data.view(torch.uint8)[::3, :, 1] = 0
    check_attention(st)
    st.scales[:, :, 1] *= 0.77                                    # scales that are no powers of two
    check_attention(st)


def test_rows_that_see_nothing_and_pages_that_are_not_there():
    st = Setup(17, [-1, 300, 70, 20], [2, 3, 2, 1], 8, 2, 64)
    st.table[1, 4], st.table[1, 9], st.table[2, 0] = -1, 12345, -7
    st.table[3, :] = -1
    out = check_attention(st)
    assert torch.all(out[-1] == 0) and torch.all(out[:2] == 0)


@pytest.mark.parametrize("hd", [64, 128])
def test_what_is_no_number_in_a_masked_place(hd):
    """A NaN among the keys or values of window token 3 reaches the rows that see it, and no other; the places behind the window hold
    NaN throughout."""
    for n, w in ((61, 6), (64, 6), (10, 40)):
        st = Setup(18, [n], [w], 4, 2, hd)
        raw = ref.page_rows(st.data, hd).view(torch.uint8)
        at = lambda pos: (int(st.table[0, pos // 32]), pos % 32)  # noqa: E731
        for pos in range(n + w, st.table.shape[1] * 32):
            raw[at(pos)[0], :, :, at(pos)[1]] = 0x7f
        st.data = ref.make_pages(raw.view(ref.F8), hd)
        q = st.randn(w, 4 * hd).to(torch.bfloat16)
        check_attention(st, q=q)
        clean = torch.empty((w, 4 * hd), dtype=torch.bfloat16, device="cuda")
        dirty = torch.empty_like(clean)
        sv.spec_kv8_attention(st.cache(), q, st.row0, st.kv_len, 4, w, 0, 0.125, clean)
        for kv in (0, 1):
            hurt = raw.clone()
            hurt[at(n + 3)[0], 0, kv, at(n + 3)[1], 5] = 0xff
            st.data = ref.make_pages(hurt.view(ref.F8), hd)
            sv.spec_kv8_attention(st.cache(), q, st.row0, st.kv_len, 4, w, 0, 0.125, dirty)
            seen = torch.zeros((w, 4, hd), dtype=torch.bool, device="cuda")
            seen[3:, :2, slice(None) if kv == 0 else slice(5, 6)] = True
            assert torch.equal(dirty.view(w, 4, hd).isnan(), seen)
            a, b = dirty.view(w, 4, hd)[~seen].float(), clean.view(w, 4, hd)[~seen].float()
            assert torch.all((a - b).abs() <= 2 * (REL * b.abs() + WEIGHTS * 4))
        st.data = ref.make_pages(raw.view(ref.F8), hd)


def test_queries_inside_the_projection_and_rows_of_no_sequence():
    st = Setup(19, [40, 50], [2, 3], 4, 2, 64)
    wide = st.randn(7, (4 + 4) * 64).to(torch.bfloat16)
    q = wide[:, : 4 * 64]
    a, b = (torch.full((7, 4 * 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = torch.empty(1 << 20, device="cuda")
    for out, x, work in ((a, q, None), (b, q.contiguous(), ws)):
        sv.spec_kv8_attention(st.cache(), x, st.row0, st.kv_len, 4, 3, 64, 0.125, out, work)
        assert torch.all(out[5:] == 7)
    assert torch.all((a.float() - b.float()).abs() <= 2 * (REL * a.float().abs() + WEIGHTS * 4))


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GiB: the pages of one sequence lie at its end."""
    st = Setup(20, [70], [2], 8, 8, 128)
    pages = (1 << 32) // (8 * 2 * 32 * 128) + 8
    data = torch.empty((pages, 8, 2, 32 * 128), dtype=torch.uint8, device="cuda").view(ref.F8)
    scales = torch.ones((pages, 8, 2), device="cuda")
    for i in range(3):
        data.view(torch.uint8)[pages - 1 - i] = st.data.view(torch.uint8)[int(st.table[0, i])]
        scales[pages - 1 - i] = st.scales[int(st.table[0, i])]
        st.table[0, i] = pages - 1 - i
    st.data, st.scales = data, scales
    sv.spec_kv8_append(st.cache(), st.qkv, st.row0, st.kv_len, 8, 2, st.cos_sin, torch.empty((2, 1024), dtype=torch.bfloat16, device="cuda"))
    check_attention(st)


def test_append_and_attention_in_a_graph_and_on_another_stream():
    st = Setup(21, [300, 40, 1500], [3, 3, 3], 8, 2, 128)
    q, out = (torch.empty((9, 8 * 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = torch.empty(1 << 22, device="cuda")
    cache = st.cache()

    def step(stream=None):
        sv.spec_kv8_append(cache, st.qkv, st.row0, st.kv_len, 8, 3, st.cos_sin, q, stream=stream)
        sv.spec_kv8_attention(cache, q, st.row0, st.kv_len, 8, 3, 2048, 0.088, out, ws, stream=stream)

    step()
    want = out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for r in range(3):
        st.qkv.mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step()
        assert torch.equal(got, out)
