"""What the compiler made of the kernels on packed prompts (no GPU): the 32 x 32 x 16 products' results are waited for longer than those of
the 16 x 16 ones, and no kernel has memory of its own."""
import re

from test_device_code import _tool, fewest_wait_states, kernels, objects  # noqa: F401

# An XDL product of eight passes: passes + 3
WAIT_STATES = 11
PRODUCT = "v_mfma_f32_32x32x16_bf16"


def test_results_of_large_products_are_waited_for(kernels):  # noqa: F811
    users = [k for k in kernels if any(op == PRODUCT for op, _ in k.ins)]
    assert len(users) >= 6      # two head sizes; one, two and four wavefronts
    found = [(k.name, fewest_wait_states(k)) for k in users]
    assert all(w for _, w in found)
    assert [f for f in found if f[1][0] < WAIT_STATES] == []


def test_no_private_memory(objects):  # noqa: F811
    ours = ("tiled_kernel", "skinny_kernel", "attention_kernelILi", "few_kernel", "rmsnorm_kernel", "append_kernel", "append_cover_kernel", "join_kernel")
    sizes = [m for o in objects for m in re.findall(r"\.name:\s+(_Z\S+).*?\.private_segment_fixed_size:\s+(\d+)", _tool("llvm-readelf", "--notes", o), re.S)]
    mine = [(n, size) for n, size in sizes if any(name in n for name in ours)]
    assert {name for name in ours if any(name in n for n, _ in mine)} == set(ours)
    assert [m for m in mine if m[1] != "0"] == []
