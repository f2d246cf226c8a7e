"""Values close to the smallest bf16 in sequences that are cut into parts: the parts' fp16
records scale by a power of two that must stay in fp32's range."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from gpu_common import assert_close, oracle_call, wrap
from paper_2609_34538_amd import _lib as das
from paper_2609_34538_amd import datagen as dg
from q8_ref import HostCache, attention, random_cache, tolerance
from test_gpu_attn_q8 import _block

pytestmark = pytest.mark.gpu
DEV = "cuda"
SCALE = 2.0 ** -118


@pytest.mark.parametrize("dh,G,w", [(64, 1, 8), (96, 1, 33), (128, 2, 20), (64, 8, 33), (128, 4, 64)])
def test_small_block_values_over_an_8_bit_cache(dh, G, w):
    """Prefix values of 0, so that the block's alone count; to half a step of bf16, whose
    smallest is 2^-133, beside the usual bound."""
    lens = [4000, 700]
    cache, batch, table = random_cache(7, torch.bfloat16, 2, 2, dh, lens)
    codes = cache.v_pool.view(torch.uint8)
    codes.copy_(torch.where(codes & 0x7f == 0x7f, codes, 0))
    q, kb, vb = _block(11, torch.bfloat16, 2, w, 2 * G, 2, dh)
    vb *= SCALE
    out = das.attn_policy_q8(cache, batch, 0, 1, 1, q, kb, vb)
    host = HostCache(cache)
    for b in range(2):
        ref, _, a, size = attention(host, table, lens, b, 0, 0, 0, q, kb, vb)
        tol = tolerance(torch.bfloat16, ref / SCALE, a / SCALE, size, lens[b] + w, dh) + 2.0 ** -134 / SCALE
        err = np.abs(out[b].double().cpu().numpy() - ref) / SCALE
        assert (err <= tol).all(), (b, float((err / tol).max()))


@pytest.mark.parametrize("path,pps", [("balanced", 0), ("mfma", 4), ("auto", 0)])
@pytest.mark.parametrize("lens", [[40000, 64, 700], [9001]])
def test_small_values_over_a_bf16_cache(path, pps, lens):
    wl = dg.scaled(dg.WORKLOADS[3], batch=len(lens), hq=2, hkv=2, dh=96, layers=1, prefix=(0, max(lens)),
                   draft_depths=(2,), draft_widths=(16,), verify_width=16, paged_random=True)
    torch.manual_seed(3)
    cd = dg.make_cache(wl, DEV, prefix_lens=lens)
    cd.v_pool.mul_(SCALE)
    cache, batch = wrap(cd)
    q, kb, vb = dg.block_inputs(cd, 16, 2, DEV)
    vb = (vb.float() * SCALE).to(vb.dtype)
    out = das.attn_policy(cache, batch, 0, 2, wl.depth_R, q, kb, vb, path=path, pages_per_split=pps)
    ref, _ = oracle_call(cd, 0, 2, wl.depth_R, q, kb, vb, range(wl.batch))
    assert_close(out.double() / SCALE, ref / SCALE, wl.dtype, f"{path} {lens}")
