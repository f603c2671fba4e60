"""dQ of packed documents at D = 128 without a cap: two blocks share a unit at 256 registers, and nothing of the tile loop lies in scratch (tile addresses reloaded from there waited for the next tile's
transfer, 390 us for 305 at 8192 rows of 32:8 heads).  The forward kernels of both widths likewise.  Read from the code objects' notes in the library built here.  No GPU needed."""
from test_kernel_registers import kernel_notes


def test_dq_and_forward_stay_in_registers():
    kernels = {n: k for n, k in kernel_notes().items() if "attn_docs_dq_bf16_kernelILi128ELb0E" in n or "attn_docs_fwd_bf16_kernel" in n}
    assert len(kernels) == 5
    for name, k in kernels.items():
        assert k[".vgpr_count"] <= 256 and k[".vgpr_spill_count"] == 0 and k[".sgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name


def test_one_block_a_unit_spills_nothing():
    kernels = {n: k for n, k in kernel_notes().items() if "attn_docs_dkv_bf16_kernelILi128E" in n or "attn_docs_bwd_bf16_kernelILi128E" in n}
    assert len(kernels) == 4  # dK/dV, both in one; with and without a cap
    for name, k in kernels.items():
        assert k[".vgpr_count"] <= 512 and k[".vgpr_spill_count"] == 0 and k[".sgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name
