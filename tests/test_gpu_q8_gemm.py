"""The product of 8-bit rows and 8-bit weights against the same product in 64 bits."""
import pytest
import torch

import q8_ref as ref
from paper_2411_00853_amd import binding as sv

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def operands(seed, M, N, K):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((M, K), generator=g, device="cuda") * torch.exp(torch.randn((M, 1), generator=g, device="cuda"))
    w = torch.randn((N, K), generator=g, device="cuda") * torch.exp(0.5 * torch.randn((N, 1), generator=g, device="cuda"))
    return *ref.quantise_rows(x), *ref.quantise_weight(w)


def check(M, N, K, dtype, seed=1):
    q, s, w, ws = operands(seed, M, N, K)
    y = torch.full((M, N), float("nan"), dtype=DTYPES[dtype], device="cuda")
    sv.spec_q8_gemm(q, s, sv.spec_q8_pack_weight(w), ws, y)
    want, mag, top = ref.gemm(q, s, w, ws)
    # products are exact, a block's sum of 128 and the sum over blocks are fp32 in some order, two more roundings for the scales; for
    # a bf16 result a block is one fp8 matrix instruction, which drops what lies below 2^-11 of its largest product, and the result is rounded
    bound = (128 + q.shape[1] // 128 + 4) * ref.U * mag + (2.0 ** -8 * want.abs() + 2.0 ** -10 * top if dtype == "bf16" else 0)
    off = (y.double() - want).abs()
    assert torch.all(off <= 1.01 * bound + 1e-30), float((off / bound).max())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 16, 128), (2, 17, 130), (1, 4096, 4096), (5, 1000, 2048), (16, 2050, 300), (17, 500, 1024)])
def test_few_rows(M, N, K, dtype):
    check(M, N, K, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,N,K", [(33, 129, 1000), (48, 2048, 2048), (64, 4099, 640), (65, 256, 8192), (100, 1333, 1408), (128, 640, 256),
                                   (161, 2049, 512), (352, 1024, 4096)])
def test_some_rows(M, N, K, dtype):
    check(M, N, K, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,N,K", [(512, 512, 512), (777, 1111, 1000), (1024, 2176, 384), (2049, 300, 2048), (1500, 4096, 128), (513, 8200, 700)])
def test_many_rows(M, N, K, dtype):
    check(M, N, K, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,N,K", [(1, 20000, 1200), (9, 9000, 700), (3, 500, 8192), (16, 4100, 5000),      # a column tile or two a workgroup
                                   (20, 3000, 1500), (30, 6001, 1100), (20, 9000, 900), (32, 20000, 700), (25, 30000, 600),
                                   (40, 3000, 1500), (48, 6001, 1100), (33, 9000, 900), (40, 20000, 700), (45, 30000, 600),
                                   (50, 3000, 1500), (64, 6001, 1100), (57, 9000, 900), (64, 20000, 700), (60, 30000, 600),
                                   (70, 2000, 2500), (600, 2500, 1300), (900, 4000, 1290), (2048, 8192, 900)])
def test_every_launch_shape(M, N, K, dtype):
    check(M, N, K, dtype)


def test_every_row_count_up_to_a_few_tiles():
    for M in range(1, 140, 3):
        check(M, 272, 384, "fp32", M)


def test_packing_is_the_order_of_the_header():
    n, k = 37, 300
    w = torch.randint(0, 256, (n, k), dtype=torch.uint8, device="cuda")
    got = sv.spec_q8_pack_weight(w.view(ref.F8)).view(torch.uint8).reshape(3, 3, 2, 4, 16, 16)     # kb, j, h, g, n, e
    p = torch.nn.functional.pad(w, (0, 384 - k, 0, 48 - n)).reshape(3, 16, 3, 2, 4, 16)            # j, n, kb, h, g, e
    assert torch.equal(got, p.permute(2, 0, 3, 4, 1, 5))


def test_a_value_that_is_no_number_stays_in_its_row_and_column():
    M, N, K = 70, 200, 256
    q, s, w, ws = operands(3, M, N, K)
    s[1, 7] = float("nan")
    q[30, 5] = torch.tensor(float("nan"), device="cuda").to(ref.F8)
    w[150, 200] = torch.tensor(float("nan"), device="cuda").to(ref.F8)
    y = torch.empty((M, N), device="cuda")
    sv.spec_q8_gemm(q, s, sv.spec_q8_pack_weight(w), ws, y)
    bad = torch.zeros((M, N), dtype=torch.bool, device="cuda")
    bad[7] = bad[30] = True
    bad[:, 150] = True
    assert torch.equal(y.isnan(), bad)


def test_on_a_stream_of_its_own_and_in_a_graph():
    for M in (3, 50, 600):
        q, s, w, ws = operands(4, M, 512, 640)
        p = sv.spec_q8_pack_weight(w)
        y = torch.empty((M, 512), device="cuda")
        want = sv.spec_q8_gemm(q, s, p, ws, torch.empty_like(y)).clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        sv.spec_q8_gemm(q, s, p, ws, y, stream=side)
        side.synchronize()
        assert torch.equal(y, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sv.spec_q8_gemm(q, s, p, ws, y)
        for r in range(3):
            s.mul_(1.5)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, sv.spec_q8_gemm(q, s, p, ws, torch.empty_like(y)))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,N", [(130, 4000), (350, 4090), (1024, 4096), (2047, 4100), (2040, 8190), (33, 25000), (60, 9000)])
@pytest.mark.parametrize("K", [100, 250, 380, 500, 640, 770, 896])
def test_a_few_blocks_of_k(M, N, K, dtype):
    """As many blocks as the kernels fetch ahead, fewer and more."""
    check(M, N, K, dtype)
