"""Arguments that the operators on packed prompts refuse, before any launch (no GPU needed)."""
import ctypes as C

import pytest

from paper_2411_00853_amd import binding as sv

P = C.c_void_p(4096)      # never dereferenced
ODD = C.c_void_p(4104)
INVALID, SHAPE = -1, -2
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    return sv.lib()


def refused(rc, want, lib, word):
    assert rc == want and word.encode() in lib.spec_last_error(), (rc, lib.spec_last_error())


def test_norm(lib):
    def call(x=P, t=0, ld=8, gain=P, eps=1e-5, rows=1, cols=8, y=P):
        return lib.spec_prompt_rmsnorm(x, t, ld, gain, eps, rows, cols, y, None)

    for k in ("x", "gain", "y"):
        refused(call(**{k: None}), INVALID, lib, "null")
    refused(call(t=2), INVALID, lib, "type")
    refused(call(ld=7), INVALID, lib, "apart")
    refused(call(rows=-1), INVALID, lib, "rows")
    refused(call(cols=0), INVALID, lib, "columns")
    refused(call(cols=65537, ld=70000), SHAPE, lib, "65537")
    refused(call(rows=(1 << 20) + 1), SHAPE, lib, "rows")
    for eps in (-1.0, NAN):
        refused(call(eps=eps), INVALID, lib, "eps")
    assert call(rows=0, x=None, gain=None, y=None) == 0


def test_product(lib):
    def call(x=P, ld_x=64, w=P, bias=None, residual=None, ld_r=48, rt=0, act=0, y=P, yt=0, ld_y=48, M=2, N=48, K=64, ws=None, n=0, plain=False):
        e = sv.spec_prompt_epilogue(bias, residual, ld_r, rt, act)
        return lib.spec_prompt_gemm(x, ld_x, w, None if plain else C.byref(e), y, yt, ld_y, M, N, K, ws, n, None)

    for k in ("x", "w", "y"):
        refused(call(**{k: None}), INVALID, lib, "null")
        refused(call(plain=True, **{k: None}), INVALID, lib, "null")
    for k in ("x", "w", "ws"):
        refused(call(**{k: ODD}), INVALID, lib, "aligned")
    for k in ("y", "bias", "residual"):
        refused(call(**{k: C.c_void_p(4097)}), INVALID, lib, "aligned")
    refused(call(yt=2), INVALID, lib, "type 2")
    refused(call(residual=P, rt=5), INVALID, lib, "type 5")
    for act in (-1, 5):
        refused(call(act=act), INVALID, lib, "activation")
    refused(call(M=-1), INVALID, lib, "M")
    refused(call(N=0), INVALID, lib, "N")
    refused(call(K=0), INVALID, lib, "K")
    refused(call(K=40), SHAPE, lib, "multiple of 32")
    refused(call(act=4, N=40), SHAPE, lib, "multiple of 16")
    refused(call(ld_x=56), INVALID, lib, "apart")
    refused(call(ld_x=68), INVALID, lib, "apart")
    refused(call(ld_x=(1 << 22) + 8), INVALID, lib, "apart")
    refused(call(ld_y=47), INVALID, lib, "apart")
    refused(call(residual=P, ld_r=47), INVALID, lib, "apart")
    refused(call(residual=P, ld_r=50), INVALID, lib, "residual is y")
    refused(call(residual=P, rt=1), INVALID, lib, "residual is y")
    refused(call(N=(1 << 23) + 1, ld_y=1 << 24), SHAPE, lib, "at most")
    refused(call(M=1 << 27), SHAPE, lib, "too many")
    assert call(M=0, x=None, w=None, y=None) == 0
    assert lib.spec_prompt_gemm_workspace_bytes(0, 48, 64, 0) == 0 and lib.spec_prompt_gemm_workspace_bytes(5, -1, 64, 0) == 0


def test_append_needs_a_handle(lib):
    refused(lib.spec_prompt_append(None, 0, P, 64, P, 64, P, P, None, 1, 1, None), INVALID, lib, "NULL handle")


def test_attention(lib):
    def call(ws=None, n=0, **change):
        a = sv.spec_prompt_attn_args(4096, 4096, 4096, 512, 128, 128, 512, 4096, None, 8, 2, 64, 3, 10, 10, 0, 0, 0.125, 4096)
        for k, v in change.items():
            assert hasattr(a, k)
            setattr(a, k, v)
        return lib.spec_prompt_attention(C.byref(a), ws, n, None)

    refused(lib.spec_prompt_attention(None, None, 0, None), INVALID, lib, "NULL")
    for k in ("q", "k", "v", "out", "q_row0"):
        refused(call(**{k: None}), INVALID, lib, "null")
    for k in ("q", "k", "v", "out"):
        refused(call(**{k: 4104}), INVALID, lib, "aligned")
    refused(call(ws=ODD), INVALID, lib, "aligned")
    refused(call(n_q_heads=9), INVALID, lib, "heads")
    refused(call(n_kv_heads=0), INVALID, lib, "heads")
    refused(call(head_dim=96), SHAPE, lib, "head_dim")
    refused(call(batch=-1), INVALID, lib, "sequences")
    refused(call(batch=65537), INVALID, lib, "sequences")
    refused(call(q_rows=-1), INVALID, lib, "rows")
    refused(call(k_rows=-1), INVALID, lib, "rows")
    refused(call(max_q_len=-1), INVALID, lib, "lengths")
    for s in (NAN, INF, -INF):
        refused(call(scale=s), INVALID, lib, "scale")
    for k in ("ld_q", "ld_k", "ld_v", "ld_out"):
        refused(call(**{k: 120}), INVALID, lib, "apart")
        refused(call(**{k: 516}), INVALID, lib, "apart")
        refused(call(**{k: (1 << 22) + 8}), INVALID, lib, "apart")
    refused(call(q_rows=1 << 30), SHAPE, lib, "too many")
    refused(call(n_q_heads=1024, n_kv_heads=1024, batch=65536, ld_q=65536, ld_k=65536, ld_v=65536, ld_out=65536), SHAPE, lib, "too many")
    assert call(q_rows=0) == 0 and call(batch=0) == 0
    assert lib.spec_prompt_attention_workspace_bytes(0, 1, 8, 2, 64) == 0 and lib.spec_prompt_attention_workspace_bytes(4, 1, 8, 3, 64) == 0
