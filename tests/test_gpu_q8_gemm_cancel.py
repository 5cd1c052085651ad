"""The 8-bit product where its terms cancel: an fp32 result is a sum in fp32, a bf16 result's blocks are off by up to 2^-10 of the sum of the
magnitudes of their products, as the header says."""
import pytest
import torch

import q8_ref as ref
from paper_2411_00853_amd import binding as sv

pytestmark = pytest.mark.gpu

SHAPES = [(1, 300, 640), (7, 12000, 500), (20, 3000, 1500), (48, 20000, 700), (60, 9000, 900), (130, 4000, 640), (600, 2500, 1300), (2048, 8192, 900)]


def check(q, s, w, ws, dtype):
    M, N = q.shape[0], w.shape[0]
    y = torch.full((M, N), float("nan"), dtype=dtype, device="cuda")
    sv.spec_q8_gemm(q, s, sv.spec_q8_pack_weight(w), ws, y)
    want, mag, _ = ref.gemm(q, s, w, ws)
    # fp32: 128 products of a block, the blocks, two roundings for the scales.  bf16: a block's products are cut off at 2^-13 of the largest of eight
    # neighbours, seven of them, which is less than 2^-10 of the sum of the eight; the rest as before, and the result's rounding
    bound = (128 + q.shape[1] // 128 + 4) * ref.U * mag + 1e-30
    if dtype == torch.bfloat16:
        bound = bound + 2.0 ** -10 * mag + 2.0 ** -8 * want.abs()
    off = (y.double() - want).abs()
    assert torch.all(off <= bound), float((off / bound).max())
    return y, want, mag


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_pairs_that_cancel(M, N, K, dtype):
    g = torch.Generator(device="cuda").manual_seed(M)
    r = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    x, w = r(M, K) * torch.exp(r(M, 1)), r(N, K)
    x[:, 1::2] = x[:, ::2]
    w[:, 1::2] = -w[:, ::2]
    w[:, ::26] = 0.01 * r(N, w[:, ::26].shape[1])          # what is left of the sum
    _, want, mag = check(*ref.quantise_rows(x), *ref.quantise_weight(w), dtype)
    assert float((want.abs() / mag).median()) < 0.2


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_many_small_products_beside_large_ones_that_cancel(M, N, K, dtype):
    """One large product in eight, of either sign in turn, and seven small ones of one sign."""
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.rand((M, K), generator=g, device="cuda") * 0.01 + 0.01
    w = torch.rand((N, K), generator=g, device="cuda") * 0.01 + 0.01
    x[:, ::8], w[:, ::16], w[:, 8::16] = 1.0, 1.0, -1.0
    check(*ref.quantise_rows(x), *ref.quantise_weight(w), dtype)


@pytest.mark.parametrize("M", [1, 20, 60, 130, 600])
def test_an_fp32_result_keeps_what_is_left(M):
    """448 * 448 - 448 * 448 + 2^-4, exactly in whatever order: no partial sum reaches 2^19, below which fp32 has every multiple of 2^-5.  (The
    fp8 instruction would drop it: it is 2^-22 of the others.)"""
    x, w = torch.zeros((M, 256), device="cuda"), torch.zeros((500, 256), device="cuda")
    x[:, 3], x[:, 4], x[:, 5], w[:, 3], w[:, 4], w[:, 5] = 448, 448, 0.25, 448, -448, 0.25
    one = torch.ones((2, M), device="cuda"), torch.ones((4, 2), device="cuda")
    y = torch.empty((M, 500), device="cuda")
    sv.spec_q8_gemm(x.to(ref.F8), one[0], sv.spec_q8_pack_weight(w.to(ref.F8)), one[1], y)
    assert torch.all(y == 2.0 ** -4)
