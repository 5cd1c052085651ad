"""What the compiler made of the 8-bit products, read from the built library's disassembly (no GPU).

* The operands of a 16x16x128 product are eight registers each.  Where such operands are carried round a loop, the compiler has
  placed a product's result over an operand that a later product still read: the sums were wrong for some tile shapes only.
  The source hides each operand's origin from the compiler (Block<uint16_t>::op); here the code is searched for what it prevents.
* Arrays of a thread are registers, not memory of its own.
* The product takes eight passes: twelve wait states before another vector instruction reads its result."""
import re

import pytest

from test_device_code import Code, _is_store, _regs, _tool, _vector, fewest_wait_states, kernels, objects  # noqa: F401

WAIT_STATES = 12


def _f8(op):
    return op.startswith("v_mfma") and "f8f6f4" in op


def overwritten_operands(code):
    """(product, reader) where a product's result covers a register of one of its operands, and a later product of the same block of
    code reads that operand again without a write to it in between."""
    found = []
    for i, (op, a) in enumerate(code.ins):
        if not _f8(op):
            continue
        for source in a[1:3]:
            lost = _regs(a[0]) & _regs(source)
            for k in range(i + 1, len(code.ins)):
                name, b = code.ins[k]
                if not lost or name.startswith(("s_branch", "s_cbranch", "s_endpgm")):
                    break
                if _f8(name):
                    if any(_regs(o) == _regs(source) for o in b[1:3]) and lost & _regs(source):
                        found.append((i, k))
                        break
                    lost = lost - _regs(b[0])
                elif _vector(name) and not _is_store(name) and b:
                    lost = lost - _regs(b[0])
    return found


def products(kernels):
    return [c for c in kernels if any(_f8(op) for op, _ in c.ins)]


def test_the_products_are_there(kernels):
    assert len(products(kernels)) >= 8
    assert any("skinny" in c.name for c in products(kernels)) and any("tiled" in c.name for c in products(kernels))


def test_no_product_overwrites_an_operand_in_use(kernels):
    bad = {c.name: overwritten_operands(c) for c in products(kernels)}
    assert not {n: f for n, f in bad.items() if f}


def test_results_of_eight_passes_are_waited_for(kernels):
    for c in products(kernels):
        assert all(_f8(op) for op, _ in c.ins if op.startswith("v_mfma")), c.name
        near = fewest_wait_states(c)
        assert near is None or near[0] >= WAIT_STATES, (c.name, near)


@pytest.mark.parametrize("between,found", (
    ([], 1),
    (["v_mov_b32_e32 v9, v0"], 0),
    (["ds_read_b128 v[8:11], v60"], 0),
    (["s_cbranch_scc1 4"], 0),
))
def test_the_search_finds_what_it_looks_for(between, found):
    lines = ["v_mfma_f32_16x16x128_f8f6f4 v[6:9], v[8:15], v[16:23], 0", *between, "v_mfma_f32_16x16x128_f8f6f4 v[40:43], v[8:15], v[24:31], 0"]
    if between and between[0].startswith("v_mov"):
        lines[1:2] = ["v_mov_b32_e32 v8, v0", between[0]]
    text = ["\t%s // %012X: 00000000" % (l, 0x100 + 8 * i) for i, l in enumerate(lines)]
    assert len(overwritten_operands(Code("f", text))) == found


def test_a_result_over_its_operand_alone_is_no_fault():
    lines = ["v_mfma_f32_16x16x128_f8f6f4 v[8:11], v[8:15], v[16:23], 0", "v_mfma_f32_16x16x128_f8f6f4 v[40:43], v[32:39], v[24:31], 0"]
    text = ["\t%s // %012X: 00000000" % (l, 0x100 + 8 * i) for i, l in enumerate(lines)]
    assert not overwritten_operands(Code("f", text))


def test_no_8_bit_or_draw_kernel_has_private_memory(objects):
    """A thread's arrays are registers.  A row of logits that a function was called with was not: it lay in memory, at half the speed."""
    ours = ("rows_kernel", "norm_kernel", "skinny_kernel", "tiled_kernel", "append_kernel", "attn8_kernel", "join_kernel", "filter_kernel", "part_")
    seen = {}
    for o in objects:
        notes = _tool("llvm-readelf", "--notes", o)
        for name, size in re.findall(r"\.name:\s+(\S+).*?\.private_segment_fixed_size:\s+(\d+)", notes, re.S):
            if any(k in name for k in ours) and "rope_append" not in name:
                seen[name] = int(size)
    assert len(seen) > 40
    assert not {n: v for n, v in seen.items() if v}
