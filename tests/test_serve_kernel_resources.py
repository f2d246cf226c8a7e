"""The kernels of the 8-bit cache, the sampler and the page tables are in the compiler's
resource report, which the checks of scratch memory and LDS go through, and the attention
keeps to the registers of two waves per SIMD."""

from test_kernel_resources import _kernels


def test_report_covers_the_serving_kernels():
    names = " ".join(k[0] for k in _kernels())
    for family in ("attn_q8_kernel", "attn_q8_combine_kernel", "kv_append_q8_kernel", "sample_kernel",
                   "pages_update_kernel", "page_slots_kernel"):
        assert family in names, family


def test_every_form_of_the_attention_keeps_its_accumulators_in_vgprs():
    found = [k for k in _kernels() if "attn_q8_kernel" in k[0]]
    # bf16: 1 and 2 row tiles, 2 with 2 and 4 row waves, at 3 head dims; fp32: the same at
    # head dim 64, no 2 tiles at 128, no 2 row waves at 96 (and there 1 tile with 4)
    assert len(found) == 4 * 3 + 4 + 3 + 3
    for name, vgpr, agpr, scratch, lds in found:
        assert agpr == 0 and vgpr <= 256 and scratch == 0, f"{name}: {vgpr} VGPRs, {agpr} AGPRs"


def test_the_commit_keeps_eight_waves_per_simd():
    found = [k for k in _kernels() if "kv_append_q8_kernelIt" in k[0]]
    assert len(found) == 3
    for name, vgpr, agpr, scratch, lds in found:
        assert vgpr + agpr <= 64, f"{name}: {vgpr} VGPRs, {agpr} AGPRs"
