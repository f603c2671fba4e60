"""The D = 64 dK/dV kernels of packed documents keep within the 256 registers that let two blocks share a unit, capped or not, and nothing of theirs lies in scratch (capped, 5000
rows on 16:4 heads, 360 us for the backward pass at 277 registers, 272 at 248; held to 256 with 24 of them spilled, long documents took 431 us for 352).  Read from
the code objects' notes in the library built here.  No GPU needed."""
from test_kernel_registers import kernel_notes


def test_two_blocks_of_short_heads_share_a_unit():
    kernels = {n: k for n, k in kernel_notes().items() if "attn_docs_" in n and "bf16_kernelILi64E" in n}
    assert len(kernels) == 8  # forward, dQ, dK/dV, both in one; with and without a cap
    for name, k in kernels.items():
        assert k[".vgpr_count"] <= 256 and k[".vgpr_spill_count"] == 0 and k[".sgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name
