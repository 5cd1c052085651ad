"""Arguments that the 8-bit operators and the filtered draw refuse, before any launch (no GPU needed)."""
import ctypes as C

import pytest

from paper_2411_00853_amd import binding as sv

P = C.c_void_p(4096)      # never dereferenced
INVALID, SHAPE = -1, -2
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    return sv.lib()


def refused(rc, want, lib, word):
    assert rc == want and word.encode() in lib.spec_last_error(), (rc, lib.spec_last_error())


def test_rows(lib):
    refused(lib.spec_q8_quantize(P, 2, 8, 1, 8, P, P, None), INVALID, lib, "type")
    refused(lib.spec_q8_quantize(P, 0, 7, 1, 8, P, P, None), INVALID, lib, "apart")
    refused(lib.spec_q8_quantize(P, 0, 8, -1, 8, P, P, None), INVALID, lib, "rows")
    refused(lib.spec_q8_quantize(P, 0, 8, 1, 0, P, P, None), INVALID, lib, "columns")
    refused(lib.spec_q8_quantize(None, 0, 8, 1, 8, P, P, None), INVALID, lib, "null")
    refused(lib.spec_q8_quantize(P, 0, 8, 1, 8, C.c_void_p(4104), P, None), INVALID, lib, "aligned")
    assert lib.spec_q8_quantize(None, 0, 8, 0, 8, None, None, None) == 0
    refused(lib.spec_q8_swiglu(P, 0, 1, 8, P, None, None), INVALID, lib, "null")
    refused(lib.spec_q8_add_rmsnorm(P, 0, None, 0, P, -1.0, 1, 8, None, P, P, None), INVALID, lib, "eps")
    refused(lib.spec_q8_add_rmsnorm(P, 0, None, 0, P, NAN, 1, 8, None, P, P, None), INVALID, lib, "eps")
    refused(lib.spec_q8_add_rmsnorm(P, 0, P, 9, P, 1e-5, 1, 8, None, P, P, None), INVALID, lib, "type")
    refused(lib.spec_q8_add_rmsnorm(P, 0, None, 0, None, 1e-5, 1, 8, None, P, P, None), INVALID, lib, "null")
    refused(lib.spec_q8_add_rmsnorm(P, 0, None, 0, P, 1e-5, 1, 65537, None, P, P, None), SHAPE, lib, "65537")


def test_product(lib):
    ok = [P, P, P, P, P, 0, 1, 16, 128, None]

    def call(**change):
        a = list(ok)
        for i, v in change.items():
            a[int(i[1:])] = v
        return lib.spec_q8_gemm(*a)

    for i in range(5):
        refused(call(**{f"a{i}": None}), INVALID, lib, "null")
    for i in (0, 2, 4):
        refused(call(**{f"a{i}": C.c_void_p(4100)}), INVALID, lib, "aligned")
    refused(call(a5=3), INVALID, lib, "type")
    refused(call(a6=-1), INVALID, lib, "M")
    refused(call(a7=0), INVALID, lib, "N")
    refused(call(a8=0), INVALID, lib, "K")
    assert call(a6=0) == 0
    refused(lib.spec_q8_pack_weight(None, P, 16, 128, None), INVALID, lib, "null")
    refused(lib.spec_q8_pack_weight(P, P, 0, 128, None), INVALID, lib, "0 x")
    refused(lib.spec_q8_pack_weight(P, C.c_void_p(4097), 16, 128, None), INVALID, lib, "aligned")
    assert sv.spec_q8_packed_weight_bytes(17, 129) == 2 * 2 * 2048 and sv.spec_q8_packed_weight_bytes(0, 5) == 0


def cache(**change):
    c = sv.spec_kv8_cache(4096, 4096, 4096, 10, 2, 64, 3, 4)
    for k, v in change.items():
        setattr(c, k, v)
    return C.byref(c)


def test_cache(lib):
    def append(c=None, qkv=P, hq=4, row0=P, kv=P, rows=3, win=1, cs=P, pos=100, q=P):
        return lib.spec_kv8_append(c or cache(), qkv, hq, row0, kv, rows, win, cs, pos, q, None)

    def attend(c=None, q=P, ld=256, hq=4, row0=P, kv=P, rows=3, win=1, most=0, scale=1.0, out=P, ws=None, n=0):
        return lib.spec_kv8_attention(c or cache(), q, ld, hq, row0, kv, rows, win, most, scale, out, ws, n, None)

    for call in (append, attend):
        refused(call(cache(head_dim=96)), SHAPE, lib, "head_dim")
        refused(call(hq=5), SHAPE, lib, "query heads")
        refused(call(win=4), SHAPE, lib, "window")
        refused(call(cache(batch=70000)), SHAPE, lib, "batch")
        for name in ("n_pages", "n_kv_heads", "batch", "blocks_per_seq"):
            refused(call(cache(**{name: 0})), INVALID, lib, "batch")
        refused(call(rows=-1), INVALID, lib, "rows")
        for name in ("data", "scales", "table"):
            refused(call(cache(**{name: None})), INVALID, lib, "null")
        refused(call(cache(data=4100)), INVALID, lib, "aligned")
        refused(call(row0=None), INVALID, lib, "null")
        refused(call(kv=None), INVALID, lib, "null")
        assert call(rows=0, win=0) == 0
    refused(append(qkv=None), INVALID, lib, "null")
    refused(append(q=None), INVALID, lib, "null")
    refused(append(pos=0), INVALID, lib, "rotation")
    refused(attend(q=None), INVALID, lib, "null")
    refused(attend(out=None), INVALID, lib, "null")
    refused(attend(ld=255), INVALID, lib, "apart")
    refused(attend(ld=248), INVALID, lib, "apart")
    refused(attend(q=C.c_void_p(4098)), INVALID, lib, "aligned")
    refused(attend(ws=C.c_void_p(4100), n=64), INVALID, lib, "aligned")
    refused(attend(most=-1), INVALID, lib, "max_len")
    for s in (NAN, INF):
        refused(attend(scale=s), INVALID, lib, "scale")
    refused(lib.spec_kv8_append(None, P, 4, P, P, 3, 1, None, 0, None, None), INVALID, lib, "cache")


def test_filtered_draw(lib):
    def call(**change):
        a = sv.spec_filter_args(4096, 0, 2, 100, 100, 4096, None, None, None, None)
        o = sv.spec_filter_out(4096, None, None, None)
        ws, n = None, 0
        for k, v in change.items():
            if k == "ws":
                ws, n = v, 1 << 20
            else:
                setattr(o if k == "tokens" else a, k, v)
        return lib.spec_filter_sample(C.byref(a), C.byref(o), ws, n, None)

    refused(call(dtype=7), INVALID, lib, "type")
    refused(call(rows=-1), INVALID, lib, "rows")
    refused(call(vocab=0), INVALID, lib, "logits")
    refused(call(ld=99), INVALID, lib, "apart")
    refused(call(vocab=262145, ld=262145), SHAPE, lib, "262145")
    for name in ("logits", "uniforms", "tokens"):
        refused(call(**{name: None}), INVALID, lib, "null")
    refused(call(ws=C.c_void_p(4100)), INVALID, lib, "aligned")
    assert call(rows=0) == 0
    assert lib.spec_filter_sample(None, None, None, 0, None) == INVALID


def test_the_binding_mirrors_the_structs(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = ("spec_kv8_cache", "spec_filter_args", "spec_filter_out")
    src = ['#include <stddef.h>', '#include <stdio.h>', '#include "spec_q8.h"', "int main(void) {"]
    for n in names:
        src.append(f'  printf("%zu\\n", sizeof({n}));')
        src += [f'  printf("%zu\\n", offsetof({n}, {f}));' for f, _ in getattr(sv, n)._fields_]
    (tmp_path / "s.c").write_text("\n".join(src + ["  return 0;", "}"]) + "\n")
    exe = str(tmp_path / "s")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(root, "include"),
                    str(tmp_path / "s.c"), "-o", exe], check=True)
    got = [int(v) for v in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for n in names:
        c = getattr(sv, n)
        want += [C.sizeof(c)] + [getattr(c, f).offset for f, _ in c._fields_]
    assert got == want


def test_tensors_that_are_not_on_the_device():
    """The binding reads no address of a host tensor."""
    import torch
    x, q, s = torch.zeros(2, 128), torch.zeros((2, 128), dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros(1, 2)
    i, b = torch.zeros(3, dtype=torch.int32), torch.zeros((2, 256), dtype=torch.bfloat16)
    sv._raw_stream, keep = (lambda stream: None), sv._raw_stream
    try:
        cache = sv.Kv8Cache(q, s, i, 64)
        for call in (lambda: sv.spec_q8_quantize(x, q, s), lambda: sv.spec_q8_add_rmsnorm(x, None, s, 1e-5, None, q, s),
                     lambda: sv.spec_q8_swiglu(x, q, s), lambda: sv.spec_q8_gemm(q, s, q, s, x),
                     lambda: sv.spec_kv8_append(cache, b, i, i, 4, 1), lambda: sv.spec_kv8_attention(cache, b, i, i, 4, 1, 0, 1.0, b),
                     lambda: sv.spec_filter_sample(x, s, None, i)):
            with pytest.raises(ValueError, match="device tensor"):
                call()
        with pytest.raises(ValueError, match="expected a tensor"):
            sv.spec_filter_sample([1.0], s, None, i)
    finally:
        sv._raw_stream = keep
