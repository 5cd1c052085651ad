"""Workspaces for any number of rows up to one: few rows share out what many do not (no GPU needed)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2411_00853_amd import binding as sv
from paper_2411_00853_amd import workload as wl
from paper_2411_00853_amd.prompt import Prompt

SMALL = wl.ModelShape(2, 384, 6, 2, 64, 640, 1000)


@pytest.mark.parametrize("shape,rows,batch", [(wl.SEVEN_B, 4096, 1), (wl.SEVEN_B, 3328, 4), (wl.SEVEN_B_DRAFT, 1000, 8), (SMALL, 700, 40)])
def test_a_pass_of_fewer_rows_than_there_is_room_for_has_the_workspace_it_asks_for(shape, rows, batch):
    """Every product of the pass, and its attention, of up to `rows` rows of up to `batch` prompts."""
    cfg = sv.make_cfg(shape, batch, 64, 0)
    work = Prompt(SimpleNamespace(cfg=cfg), {"tok_embed": torch.empty(1)}, rows).work.numel()
    hd, d = shape.head_dim, shape.d_model
    most = 0
    for r in {1, 2, 17, 37, 100, 128, 300, 512, 1000, 1024, 2048, rows}:
        if r > rows:
            continue
        need = [sv.spec_prompt_gemm_workspace_bytes(r, (shape.n_q_heads + 2 * shape.n_kv_heads) * hd, d),
                sv.spec_prompt_gemm_workspace_bytes(r, d, shape.n_q_heads * hd), sv.spec_prompt_gemm_workspace_bytes(r, shape.d_ffn, d, "swiglu"),
                sv.spec_prompt_gemm_workspace_bytes(r, d, shape.d_ffn)]
        need += [sv.spec_prompt_gemm_workspace_bytes(b, shape.vocab, d) for b in range(1, batch + 1)]
        need += [sv.spec_prompt_attention_workspace_bytes(r, b, shape.n_q_heads, shape.n_kv_heads, hd) for b in range(1, batch + 1)]
        assert max(need) <= work, r
        most = max(most, *need)
    assert most > 1 << 16      # (that some of them want one)
    assert work <= 1 << 28


@pytest.mark.parametrize("N,K,act", [(4096, 4096, "none"), (4096, 11008, "none"), (11008, 4096, "swiglu"), (100, 32, "none"), (384, 640, "relu"), (32000, 4096, "none"),
                                     (17, 100000 // 32 * 32, "none")])
def test_products_of_up_to_some_rows(N, K, act):
    """The need of the numbers below, the largest of them exactly."""
    need = [0] + [sv.spec_prompt_gemm_workspace_bytes(m, N, K, act) for m in range(1, 1200)]
    for rows in (1, 16, 17, 33, 64, 100, 257, 640, 1199):
        assert sv.spec_prompt_gemm_workspace_bytes_up_to(rows, N, K, act) == max(need[:rows + 1])
    top = sv.spec_prompt_gemm_workspace_bytes_up_to(1 << 20, N, K, act)
    assert sv.spec_prompt_gemm_workspace_bytes_up_to((1 << 31) - 1, N, K, act) == top      # (more rows than a call takes ask for nothing)
    assert top >= max(need) and top <= 1 << 27
    assert all(sv.spec_prompt_gemm_workspace_bytes(m, N, K, act) <= top for m in range(1200, 1 << 20, 4999))


@pytest.mark.parametrize("hq,hk,hd", [(32, 32, 128), (32, 8, 64), (8, 1, 128), (6, 2, 64), (1, 1, 64), (71, 1, 64), (512, 512, 64)])
def test_attention_of_up_to_some_rows_and_sequences(hq, hk, hd):
    need = sv.spec_prompt_attention_workspace_bytes
    for rows, batch in ((1, 1), (40, 3), (300, 300), (2000, 1), (2000, 40), (9000, 8)):
        top = sv.spec_prompt_attention_workspace_bytes_up_to(rows, batch, hq, hk, hd)
        rs = sorted({1, 2, 3, 5, 8, 9, 16, 17, 31, 33, 64, 65, 127, 129, 200, 333, 511, 513, 999, 1500, 4000, 7777, rows})
        assert all(need(r, b, hq, hk, hd) <= top for r in rs if r <= rows for b in range(1, batch + 1, max(1, batch // 50)))
        # no more than twice a unit of partial results for each place of a workgroup of one wavefront, or two thirds as many of twice the rows
        assert top <= 2 * 4096 * 32 * (hd + 2) * 4


def test_nothing_for_calls_that_are_refused():
    product, attention = sv.spec_prompt_gemm_workspace_bytes_up_to, sv.spec_prompt_attention_workspace_bytes_up_to
    assert product(0, 48, 64) == product(5, -1, 64) == product(5, 48, 0) == product(5, (1 << 23) + 1, 64) == 0
    assert attention(0, 1, 8, 2, 64) == attention(4, 0, 8, 2, 64) == attention(4, 1, 8, 3, 64) == attention(4, 1, 8, 2, 96) == 0
