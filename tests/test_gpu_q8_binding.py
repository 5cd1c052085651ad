"""What the binding of the 8-bit calls refuses of a tensor: its type, shape and strides."""
import pytest
import torch

import q8_ref as ref
from paper_2411_00853_amd import binding as sv

pytestmark = pytest.mark.gpu


def z(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype, device="cuda")


def f8(*shape):
    return z(*shape, dtype=torch.uint8).view(ref.F8)


BF, I = torch.bfloat16, torch.int32


def refused(match, call):
    with pytest.raises(ValueError, match=match):
        call()


def test_rows():
    refused("Float or BFloat16", lambda: sv.spec_q8_quantize(z(2, 128, dtype=torch.float16), f8(2, 128), z(1, 2)))
    refused("scales: expected shape", lambda: sv.spec_q8_quantize(z(2, 200), f8(2, 256), z(2, 3)))
    refused("q: expected shape", lambda: sv.spec_q8_quantize(z(2, 200), f8(2, 200), z(2, 2)))
    refused("q: expected Float8", lambda: sv.spec_q8_quantize(z(2, 128), z(2, 128), z(1, 2)))
    refused("contiguous elements", lambda: sv.spec_q8_quantize(z(128, 2).t(), f8(2, 128), z(1, 2)))
    refused("two dimensions", lambda: sv.spec_q8_quantize(z(128), f8(2, 128), z(1, 2)))
    refused("up columns", lambda: sv.spec_q8_swiglu(z(2, 255), f8(2, 128), z(1, 2)))
    refused("x: expected a contiguous", lambda: sv.spec_q8_add_rmsnorm(z(2, 256)[:, :128], None, z(128), 1e-5, None, f8(2, 128), z(1, 2)))
    refused("delta: expected shape", lambda: sv.spec_q8_add_rmsnorm(z(2, 128), z(1, 128), z(128), 1e-5, None, f8(2, 128), z(1, 2)))
    refused("x_out: expected Float", lambda: sv.spec_q8_add_rmsnorm(z(2, 128), None, z(128), 1e-5, z(2, 128, dtype=BF), f8(2, 128), z(1, 2)))
    refused("eps: expected a number", lambda: sv.spec_q8_add_rmsnorm(z(2, 128), None, z(128), "x", None, f8(2, 128), z(1, 2)))


def test_product():
    ok = dict(q=f8(2, 256), scales=z(2, 2), w_packed=f8(48 * 256), w_scales=z(1, 2), y=z(2, 40))
    sv.spec_q8_gemm(**ok)
    for name, bad, match in (("q", f8(2, 250), "w_packed"), ("scales", z(2, 1), "scales"), ("w_packed", f8(40 * 256), "packed matrix"),
                             ("w_scales", z(2, 2), "w_scales"), ("y", z(3, 40), "y: expected shape"), ("y", z(2, 40, dtype=I), "y: expected"),
                             ("scales", z(2, 2, dtype=BF), "scales: expected Float")):
        refused(match, lambda: sv.spec_q8_gemm(**dict(ok, **{name: bad})))


def test_cache_and_draw():
    cache = sv.Kv8Cache(f8(4, 2, 2, 32 * 64), z(4, 2, 2), z(3, 2, dtype=I), 64)
    row0, kv_len, qkv, q = z(4, dtype=I), z(3, dtype=I), z(5, 8 * 64, dtype=BF), z(5, 4 * 64, dtype=BF)
    sv.spec_kv8_append(cache, qkv, row0, kv_len, 4, 2, None, q)
    refused("data: expected shape", lambda: sv.spec_kv8_append(sv.Kv8Cache(cache.data, cache.scales, cache.table, 128), qkv, row0, kv_len, 4, 2))
    refused("qkv: expected shape", lambda: sv.spec_kv8_append(cache, qkv, row0, kv_len, 2, 2))
    refused("row0", lambda: sv.spec_kv8_append(cache, qkv, kv_len, kv_len, 4, 2))
    refused("cos_sin", lambda: sv.spec_kv8_append(cache, qkv, row0, kv_len, 4, 2, z(9, 64, 2), q))
    refused("q_out", lambda: sv.spec_kv8_append(cache, qkv, row0, kv_len, 4, 2, z(9, 32, 2), z(5, 64, dtype=BF)))
    refused("q: expected BFloat16", lambda: sv.spec_kv8_attention(cache, q.float(), row0, kv_len, 4, 2, 0, 1.0, q))
    refused("out: expected shape", lambda: sv.spec_kv8_attention(cache, q, row0, kv_len, 4, 2, 0, 1.0, q[:4]))
    with pytest.raises(sv.SpecError, match="window"):
        sv.spec_kv8_attention(cache, q, row0, kv_len, 4, 6, 0, 1.0, torch.empty_like(q))
    x, u, t = z(3, 50), z(3), z(3, dtype=I)
    refused("top_k: expected Int", lambda: sv.spec_filter_sample(x, u, None, t, z(3)))
    refused("tokens: expected shape", lambda: sv.spec_filter_sample(x, u, None, z(2, dtype=I)))
    refused("logits_out", lambda: sv.spec_filter_sample(x, u, None, t, logits_out=z(3, 49)))
