"""Registers of the 8-bit cache's built kernels (CPU): none spills, but for the chunk attention's, which set aside a
few outside their loops."""
from paper_2308_16369_amd import build
from test_kernel_resources import _code_objects, _kernels


def test_no_kernel_of_the_8_bit_cache_spills_registers():
    with open(build.LIB, "rb") as f:
        lib = f.read()
    kernels = {k[".name"]: k for elf in _code_objects(lib) for k in _kernels(elf) if "kv8_" in k[".name"]}
    # append: 4 row kinds x formats of 3 (head_dim 64) or 4 register passes; read; decodes and their join; chunks; plan rows
    for name, n in (("kv8_append", 28), ("kv8_read", 4), ("kv8_attn_rows", 8), ("kv8_join", 4), ("kv8_attn_chunk", 12),
                    ("kv8_rows_kernel", 1)):
        assert sum(name in k for k in kernels) == n, name
    spilled = {k: v[".vgpr_spill_count"] for k, v in kernels.items() if v[".vgpr_spill_count"] or v[".sgpr_spill_count"]}
    assert all("kv8_attn_chunk" in k and n <= 8 for k, n in spilled.items()), spilled
    private = {k: v[".private_segment_fixed_size"] for k, v in kernels.items() if v[".private_segment_fixed_size"]}
    assert all("kv8_attn_chunk" in k and n <= 64 for k, n in private.items()), private
