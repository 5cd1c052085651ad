"""The operators on packed prompts where sizes change what runs, strides pass 32 bits, workspaces are smaller than asked for, and calls overlap."""
import pytest
import torch

import prompt_ref as ref
from paper_2411_00853_amd import binding as sv

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
FAR = 1 << 22       # elements from a row to the next, the most there may be: 600 rows pass 2^31 elements and 2^32 bytes


def far(rows, cols, dtype=BF16, at=0):
    """rows x cols with rows FAR elements apart; what lies between is not initialised."""
    return torch.empty((rows * FAR,), dtype=dtype, device="cuda").as_strided((rows, cols), (FAR, 1), at)


def attend(q, k, v, hq, hk, q_lens, k_lens, out, ws=None, stream=None, **hints):
    sv.spec_prompt_attention(q, k, v, hq, hk, ref.ints(ref.starts(q_lens)), out, 0.125, k_row0=ref.ints(ref.starts(k_lens)), workspace=ws, stream=stream, **hints)


def close(got, q, k, v, hk, q_lens, k_lens):
    want, mags, big = ref.attend(q, k, v, hk, 0.125, q_lens, k_lens)
    return bool(torch.all((got.double() - want).abs() <= ref.attention_tolerance(want, mags, big, k.shape[1] // hk)))


@pytest.mark.parametrize("M,N,K", [(409, 26066, 256), (214, 22876, 256), (133, 22069, 256), (303, 16390, 256), (4912, 1595, 320), (8667, 135, 256), (17, 17, 256),
                                   (18, 17, 288), (18, 17, 384), (4122, 135, 6432), (5526, 69, 3008), (97, 17056, 3616), (25, 17, 1760), (18, 16, 1248)])
def test_product_in_every_tile(M, N, K):
    """Numbers up to 8: sums below 64 K < 2^19 are exact, however K is shared out."""
    x, w = ref.small_ints(1, M, K), ref.small_ints(2, N, K)
    packed, want = ref.pack(w), ref.product(x, w)
    n = sv.spec_prompt_gemm_workspace_bytes(M, N, K, "none")
    for size in {0, n // 2 & ~15, max(0, n - 16), n, n + 64}:       # less than asked for: fewer parts
        ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda") if size else None
        y = torch.full((M, N), 7.0, device="cuda")
        sv.spec_prompt_gemm(x, packed, y, workspace=ws)
        assert torch.equal(y.double(), want), size


@pytest.mark.parametrize("M,N,K", [(16, 200, 96), (600, 80, 64), (600, 333, 416)])
def test_product_of_rows_far_apart(M, N, K):
    x, y, r = far(M, K), far(M, N, F32, 3), far(M, N, BF16, 8)
    x.copy_(ref.small_ints(1, M, K))
    r.copy_(ref.small_ints(2, M, N))
    w = ref.small_ints(3, N, K)
    sv.spec_prompt_gemm(x, ref.pack(w), y, residual=r)
    assert torch.equal(y.double(), ref.product(x, w, residual=r))


def test_norm_of_rows_far_apart():
    x, gain = far(600, 513, BF16), ref.normal(2, 513)
    x.copy_(ref.normal(1, 600, 513, dtype=BF16))
    y = torch.empty((600, 513), dtype=BF16, device="cuda")
    sv.spec_prompt_rmsnorm(x, gain, 1e-5, y)
    v = x.double()
    want = v / (v.pow(2).mean(-1, keepdim=True) + 1e-5).sqrt() * gain.double()
    assert torch.all((y.double() - want).abs() <= want.abs() * (ref.HALF_BF16 + 2.0 ** -14))     # (513 squares: 513 2^-24, half of that in the root)


@pytest.mark.parametrize("q_lens,k_lens", [([600], [600]), ([1, 1], [590, 10]), ([40], [600])])
def test_attention_of_rows_far_apart(q_lens, k_lens):
    hq, hk, hd = 4, 2, 64
    q, k, v, out = far(sum(q_lens), hq * hd), far(sum(k_lens), hk * hd, at=8), far(sum(k_lens), hk * hd), far(sum(q_lens), hq * hd, at=16)
    for i, t in enumerate((q, k, v)):
        t.copy_(ref.normal(i, *t.shape, dtype=BF16))
    attend(q, k, v, hq, hk, q_lens, k_lens, out)
    assert close(out, q, k, v, hk, q_lens, k_lens)


def test_append_of_rows_far_apart():
    hq, hk, hd, n = 4, 2, 64, 520
    h, _, _ = ref.handle(hq=hq, hk=hk, hd=hd, slots=1, max_kv=n)
    values = ref.normal(1, n, (hq + 2 * hk) * hd, dtype=BF16)
    near, qkv, rotated = values.clone(), far(n, (hq + 2 * hk) * hd), far(n, (hq + hk) * hd, at=8)
    qkv.copy_(values)
    row0, slot = ref.ints([0, n]), ref.ints([0])
    sv.spec_prompt_append(h, 0, qkv, rotated, row0, slot)
    sv.spec_prompt_append(h, 0, near, near[:, :(hq + hk) * hd], row0, slot)
    assert torch.equal(rotated, near[:, :(hq + hk) * hd]) and torch.equal(qkv, values)


@pytest.mark.parametrize("hq,hk,hd", [(16, 16, 128), (16, 8, 64), (40, 40, 64)])
@pytest.mark.parametrize("lens", [[900, 1, 0, 700, 333, 333, 64], [(37 * i) % 150 for i in range(131)], [1000] * 5])
def test_more_tiles_than_places(hq, hk, hd, lens):
    """Many sequences of different lengths, more than 64 of them too: every tile is computed, by whichever workgroup."""
    rows = sum(lens)
    q, k, v = (ref.normal(i, rows, h * hd, dtype=BF16) for i, h in enumerate((hq, hk, hk)))
    out = torch.full_like(q, 7.0)
    attend(q, k, v, hq, hk, lens, lens, out, max_q_len=max(lens), max_k_len=max(lens))
    assert close(out, q, k, v, hk, lens, lens)


@pytest.mark.parametrize("share", (0.02, 0.1, 0.5, 1.0))
@pytest.mark.parametrize("q_lens,k_lens", [([1], [9000]), ([3, 1], [5000, 900]), ([60], [7000])])
def test_attention_with_less_workspace(share, q_lens, k_lens):
    hq, hk, hd = 8, 2, 64
    q, k, v = ref.normal(1, sum(q_lens), hq * hd, dtype=BF16), ref.normal(2, sum(k_lens), hk * hd, dtype=BF16), ref.normal(3, sum(k_lens), hk * hd, dtype=BF16)
    n = sv.spec_prompt_attention_workspace_bytes(sum(q_lens), len(q_lens), hq, hk, hd)
    size = int(n * share) & ~15
    ws = torch.full((n + 4096,), 255, dtype=torch.uint8, device="cuda")
    out = torch.full_like(q, 7.0)
    attend(q, k, v, hq, hk, q_lens, k_lens, out, ws[:size], max_q_len=max(q_lens), max_k_len=max(k_lens))
    assert close(out, q, k, v, hk, q_lens, k_lens)
    assert torch.all(ws[size:] == 255)      # nothing behind what was given


def test_calls_at_once_on_two_streams():
    """With workspaces of their own they do not disturb each other."""
    hq, hk, hd, M, N, K = 8, 2, 128, 21, 700, 4096
    x, w = ref.small_ints(1, M, K), ref.small_ints(2, N, K)
    packed, want = ref.pack(w), ref.product(x, w)
    q, k, v = ref.normal(1, 2, hq * hd, dtype=BF16), ref.normal(2, 9000, hk * hd, dtype=BF16), ref.normal(3, 9000, hk * hd, dtype=BF16)
    streams = [torch.cuda.Stream() for _ in range(2)]
    space = [[torch.full((max(16, n),), 255, dtype=torch.uint8, device="cuda") for n in (sv.spec_prompt_gemm_workspace_bytes(M, N, K, "none"),
                                                                                      sv.spec_prompt_attention_workspace_bytes(2, 1, hq, hk, hd))] for _ in streams]
    q0, k0 = ref.ints([0, 2]), ref.ints([0, 9000])
    y = [torch.zeros((20, M, N), device="cuda") for _ in streams]
    o = [torch.zeros((20, 2, hq * hd), dtype=BF16, device="cuda") for _ in streams]
    torch.cuda.synchronize()
    for i in range(20):
        for j, s in enumerate(streams):
            sv.spec_prompt_gemm(x, packed, y[j][i], workspace=space[j][0], stream=s)
            sv.spec_prompt_attention(q, k, v, hq, hk, q0, o[j][i], 0.125, k_row0=k0, max_q_len=2, max_k_len=9000, workspace=space[j][1], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(t.double(), want) for ys in y for t in ys)
    assert all(torch.equal(t, o[0][0]) for os in o for t in os) and close(o[0][0], q, k, v, hk, [2], [9000])


@pytest.mark.parametrize("act", ("none", "swiglu"))
@pytest.mark.parametrize("M", (17, 31, 32, 33))
@pytest.mark.parametrize("N,K", [(4096, 2048), (4112, 2048), (4096, 2080), (48, 1056), (4080, 32)])
def test_products_at_the_edge_between_the_kernels(act, M, N, K):
    x, w = ref.small_ints(1, M, K), ref.small_ints(2, N if act == "none" else 2 * N, K)
    y = torch.full((M, N), 7.0, device="cuda")
    ws = torch.full((max(16, sv.spec_prompt_gemm_workspace_bytes(M, N, K, act)),), 255, dtype=torch.uint8, device="cuda")
    sv.spec_prompt_gemm(x, ref.pack(w, act == "swiglu"), y, activation=act, workspace=ws)
    want = ref.product(x, w, act=act)
    if act == "none":
        assert torch.equal(y.double(), want)
    else:
        # Both products are exact, gate g and up.  exp(-g) = 2^t with t = g * -1.44269504: that constant is off by less than 2^-25 of it, the product by
        # 2^-24, so t by |g| 1.4427 * 1.5 * 2^-24 and 2^t by |g| 1.5 * 2^-24 of itself, which is less than |g| 2^-23; where g is negative the result is off
        # by as much.  The exponential, the sum, the reciprocal and two products: some 2^-20.  Below 2^-126 the reciprocal is zero: 90 * 2^-126 * 2^17 < 1e-30.
        gate = ref.product(x, w[:N])
        assert torch.all((y.double() - want).abs() <= want.abs() * (2.0 ** -20 + gate.abs() * 2.0 ** -23) + 1e-30)
