"""The kernels of the 4-bit cache, the norm and rotation and the sampled verification are in
the compiler's resource report, and none keeps anything in scratch memory."""

from test_kernel_resources import _kernels

FAMILIES = ("attn_q4_kernel", "attn_q4_combine_kernel", "kv_q4_kernel", "qk_rope_kernel",
            "accept_stats_kernel", "accept_chain_kernel", "accept_draw_kernel")


def test_report_covers_the_kernels():
    names = " ".join(k[0] for k in _kernels())
    for family in FAMILIES:
        assert family in names, family


def test_registers_and_scratch():
    for name, vgpr, agpr, scratch, lds in _kernels():
        if any(f in name for f in FAMILIES):
            assert agpr == 0 and vgpr <= 256 and scratch == 0, f"{name}: {vgpr} VGPRs, {agpr} AGPRs, {scratch} B"
