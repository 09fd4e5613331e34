"""Registers of the microscaled operators' built kernels (CPU): no loop of theirs goes to memory for one."""
from paper_2308_16369_amd import build
from test_kernel_resources import _code_objects, _kernels


def test_no_kernel_of_the_microscaled_operands_spills_registers():
    with open(build.LIB, "rb") as f:
        lib = f.read()
    kernels = {k[".name"]: k for elf in _code_objects(lib) for k in _kernels(elf) if "mx_" in k[".name"]}
    # quantise and dequantise: 2 dtypes x 2 formats; norm: 3 type pairs x 2 formats x 7 widths; block shapes of the tiles x
    # SwiGLU or not: 6 of e2m1 rows, 5 of e4m3, 4 with exact sums
    for name, n in (("mx_quantize_kernel", 4), ("mx_dequantize_kernel", 4), ("mx_norm_kernel", 42), ("mx_tile_kernel", 30),
                    ("mx_join_kernel", 1)):
        assert sum(name in k for k in kernels) == n, name
    spilled = {k: v[".vgpr_spill_count"] for k, v in kernels.items() if v[".vgpr_spill_count"] or
               v[".private_segment_fixed_size"]}
    assert not spilled, spilled
