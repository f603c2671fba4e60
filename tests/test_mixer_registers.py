"""The tile loops of window and linear attention keep what they use in registers: a register in scratch is reloaded behind the next tile's transfer, in one counter of loads, so that
every tile waits for it (window attention's dQ, D = 128: a training step of 8192 tokens on 32:8 heads 759 us with masks in scratch, 703 without; linear attention's results 78 and 60 us for
8192 tokens x 32 heads).  Read from the code objects' notes in the library built here.  No GPU needed."""
from test_kernel_registers import kernel_notes


def test_nothing_of_a_loop_lies_in_scratch():
    kernels = {n: k for n, k in kernel_notes().items() if ("attn_window_" in n and "bf16_kernelILi" in n) or "lin_fwd_kernelILi" in n or "lin_bwd_" in n}
    assert len(kernels) == 8 + 10 + 6  # forward, dQ, dK/dV, both in one; sums and results (whole rows or pieces, one team or two); sums and dK/dV (whole rows or pieces); each at two widths
    for name, k in kernels.items():
        if "lin_bwd_kernelILi128ELb1E" in name:  # whole rows whose dstate_in is asked for
            assert k[".vgpr_spill_count"] <= 3, name
        else:
            assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name


def test_waves_that_share_a_simd():
    for name, k in kernel_notes().items():
        two = "lin_fwd_kernelILi" in name or "lin_bwd_" in name or "attn_window_fwd_bf16" in name or "attn_window_dq_bf16" in name or ("attn_window_" in name and "bf16_kernelILi64E" in name)
        if two:
            assert k[".vgpr_count"] <= 256, name
