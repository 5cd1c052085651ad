"""Attention over pages whose value scales are far apart: the sum of weights has every page in it, the result what is left of each."""
import pytest
import torch

import q8_ref as ref
from paper_2411_00853_amd import binding as sv
from test_gpu_kv8 import REL, WEIGHTS, Setup

pytestmark = pytest.mark.gpu

SHAPES = [([95], [1], 4, 4, 64), ([700, 60], [2, 6], 8, 1, 128), ([3000, 1], [1, 5], 8, 2, 64), ([5000], [3], 32, 8, 128), ([900], [40], 4, 1, 128)]


def setup(lens, win, hq, hk, hd, exponents, seed=41):
    """Page i of a sequence has value scale 2^exponents[i % n]; keys as they come."""
    st = Setup(seed, lens, win, hq, hk, hd, spread=0.0)
    for b in range(len(lens)):
        for i, page in enumerate(st.table[b].tolist()):
            if page >= 0:
                st.scales[page, :, 1] = 2.0 ** exponents[i % len(exponents)]
    return st


def check_attention(st, workspace, scale=None, q=None):
    """Against the definition in 64 bits, the exponentials by themselves: a library's softmax has been seen to lose weights below 2^-126, on which
    results depend here."""
    rows, group = sum(st.win), st.hq // st.hk
    scale = st.hd ** -0.5 if scale is None else scale
    q = st.randn(rows, st.hq * st.hd).to(torch.bfloat16) if q is None else q
    out = torch.full((rows, st.hq * st.hd), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((sv.spec_kv8_workspace_bytes(rows, st.hq, st.hd) // 4,), float("nan"), device="cuda") if workspace else None
    cap = st.table.shape[1] * 32
    sv.spec_kv8_attention(st.cache(), q, st.row0, st.kv_len, st.hq, st.max_window, cap, scale, out, ws)
    for b, (n, w) in enumerate(zip(st.lens, st.win)):
        r0, length = int(st.row0[b]), min(n + w, cap)
        k, v, ok = st.held(b, length)
        assert bool(ok.all())
        qd = q[r0:r0 + w].double().reshape(w, st.hk, group, st.hd)
        got = out[r0:r0 + w].double().reshape(w, st.hk, group, st.hd)
        lim = torch.arange(w, device="cuda") + n
        for h in range(st.hk):
            score = (qd[:, h].reshape(-1, st.hd) @ k[:, h].t().contiguous() * scale).reshape(w, group, length)
            score = score.masked_fill(torch.arange(length, device="cuda") > lim[:, None, None], float("-inf"))
            p = torch.exp(score - score.amax(-1, keepdim=True))
            p = (p / p.sum(-1, keepdim=True)).reshape(-1, length)
            want, mag = ((p @ x).reshape(w, group, st.hd) for x in (v[:, h].contiguous(), v[:, h].abs().contiguous()))
            off, bound = (got[:, h] - want).abs(), REL * want.abs() + WEIGHTS * mag + 1e-30
            assert torch.all(off <= bound), (b, h, float((off / bound).max()))
    return out


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("exponents", [(60, -80), (-80, 60), (0, 40), (0, 41), (0, -41), (39, -39, 0), (119, -80), (-80, -80, -80, 119, 0), (100, 30, -40)])
@pytest.mark.parametrize("lens,win,hq,hk,hd", SHAPES)
def test_scales_apart(lens, win, hq, hk, hd, exponents, workspace):
    check_attention(setup(lens, win, hq, hk, hd, exponents), workspace)


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("first", [True, False])
@pytest.mark.parametrize("big", [30, 60, 119])
@pytest.mark.parametrize("hd", [64, 128])
def test_pages_of_zeros_count_in_the_sum(hd, big, first, workspace):
    """An appended page of zeros has the scale 2^-126.  Equal scores everywhere: half the weight is on zeros."""
    st = setup([8 * 256], [1], 4, 2, hd, (-126, big) if first else (big, -126))
    u = st.data.view(torch.uint8)
    for i, page in enumerate(st.table[0].tolist()):
        if (i % 2 == 0) == first:
            u[page, :, 1] = 0
    u[:, :, 0] = 0                                    # keys: every score is 0
    st.table = st.table[:, :64].contiguous()          # 64 whole pages; the window's own position has none
    out = check_attention(st, workspace)
    k, v, _ = st.held(0, 2048)
    want = v.sum(0) / 2048
    got = out.double().reshape(2, 2, hd)              # two query heads to a kv head
    assert torch.all((got - want[:, None]).abs() <= REL * want[:, None].abs() + WEIGHTS * v.abs().mean(0)[:, None])


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("exponents", [(60, -60), (119, -1), (40, -80), (-60, 60, 0)])
@pytest.mark.parametrize("lens,win,hq,hk,hd", SHAPES)
def test_scores_against_scales(lens, win, hq, hk, hd, exponents, workspace):
    """Pages of the largest scale have scores far below the others': their weight is small, what it multiplies is large, and which of the
    two decides the result differs from row to row."""
    st = setup(lens, win, hq, hk, hd, exponents)
    u = st.data.view(torch.uint8)
    u[:, :, 0] &= 0x7f                                # positive keys, but for the pages of the largest scale
    for b in range(len(lens)):
        for i, page in enumerate(st.table[b].tolist()):
            if page >= 0 and exponents[i % len(exponents)] == max(exponents):
                u[page, :, 0] |= 0x80
    for size in (0.05, 0.3, 1.0, 4.0):                # scores apart by some 2 to 2^10
        q = (st.randn(sum(win), hq * hd).abs() * size).to(torch.bfloat16)
        check_attention(st, workspace, scale=0.5, q=q)


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("exponents", [(3,), (30, -9), (100, -20)])
def test_large_scores_and_scales(exponents, workspace):
    """Scores of 10^5 and more, where the exponent of a scale is no longer exact beside a score: the value of the position that has all the
    weight comes out as it is."""
    st = setup([1500, 40], [2, 1], 4, 2, 128, exponents)
    q = (st.randn(3, 4 * 128) * 3e4).to(torch.bfloat16)
    check_attention(st, workspace, scale=1.0, q=q)
    q = (st.randn(3, 4 * 128) * 1e15).to(torch.bfloat16)
    check_attention(st, workspace, scale=1.0, q=q)


def test_what_is_no_number_beside_scales_apart():
    st = setup([600], [6], 4, 2, 64, (90, -60))
    raw = ref.page_rows(st.data, 64).view(torch.uint8)
    page, t = int(st.table[0, 603 // 32]), 603 % 32
    q = st.randn(6, 4 * 64).to(torch.bfloat16)
    for kv in (0, 1):
        hurt = raw.clone()
        hurt[page, 0, kv, t, 5] = 0x7f
        st.data = ref.make_pages(hurt.view(ref.F8), 64)
        for ws in (None, torch.empty(1 << 20, device="cuda")):
            out = torch.empty((6, 4 * 64), dtype=torch.bfloat16, device="cuda")
            sv.spec_kv8_attention(st.cache(), q, st.row0, st.kv_len, 4, 6, 0, 0.125, out, ws)
            seen = torch.zeros((6, 4, 64), dtype=torch.bool, device="cuda")
            seen[3:, :2, slice(None) if kv == 0 else slice(5, 6)] = True
            assert torch.equal(out.view(6, 4, 64).isnan(), seen)
