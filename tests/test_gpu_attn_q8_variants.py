"""Attention over the 8-bit cache on every form of its kernel: one and two row tiles a wave,
one, two and four waves with different rows, at the row counts where the form changes, in
one chunk and in several; and one-row-wave units of one chunk with more tiles than a wave
holds page ids for."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2609_34538_amd import _lib as das
from q8_ref import HostCache, attention, key_bytes, random_cache, tolerance
from test_gpu_attn_q8 import _block, _check

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32

ROWS = [(16, 1), (17, 1), (8, 4), (33, 1), (16, 4), (13, 5)]  # 16, 17, 32, 33, 64, 65 rows


@pytest.mark.parametrize("w,G", ROWS, ids=lambda x: str(x))
@pytest.mark.parametrize("dh", [64, 96, 128])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("lens", [[95, 0, 33], [1300, 0, 700]], ids=["one-chunk", "chunks"])
def test_every_row_count(dtype, dh, w, G, lens):
    cache, batch, table = random_cache(7, dtype, len(lens), 2, dh, lens, spread=1)
    q, kb, vb = _block(11, dtype, len(lens), w, 2 * G, 2, dh)
    lse = torch.full((len(lens), 2 * G, w), float("nan"), device=DEV)
    out = das.attn_policy_q8(cache, batch, 0, 1, 1, q, kb, vb, out=torch.full_like(q, float("nan")), lse=lse)
    _check(cache, batch, table, lens, q, kb, vb, out, lse)
    assert int(batch.dev_error) == 0
    assert torch.equal(out, das.attn_policy_q8(cache, batch, 0, 1, 1, q, kb, vb))


def _long(dtype):
    """13 x 16 units, enough for one chunk each, of 9000 tokens: 71 tiles a wave."""
    B, hkv, dh, S = 13, 16, 64, 9000
    cache = das.QuantCache.empty(1, hkv, 150, dh, 1, {1: 0}, {1: 0}, dtype)
    g = torch.Generator(device=DEV).manual_seed(1)
    for pool in (cache.k_pool, cache.v_pool):
        pool.copy_(torch.randn(pool.shape, generator=g, device=DEV).to(torch.float8_e4m3fn))
    table = np.stack([np.random.default_rng(b).permutation(150)[:141] for b in range(B)]).astype(np.int32)
    return cache, table, [S] * B


@pytest.mark.parametrize("w", [8, 20])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_one_row_wave_with_many_tiles(dtype, w):
    cache, table, lens = _long(dtype)
    batch = das.Batch(torch.tensor(lens, dtype=torch.int32, device=DEV), torch.as_tensor(table, device=DEV))
    assert das.workspace_bytes_q8(cache, batch, 16, w) == 256  # one chunk
    q, kb, vb = _block(2, dtype, 13, w, 16, 16, 64)
    lse = torch.empty((13, 16, w), device=DEV)
    out = das.attn_policy_q8(cache, batch, 0, 1, 1, q, kb, vb, lse=lse)
    _check(cache, batch, table, lens, q, kb, vb, out, lse, seqs=[0, 12])


@pytest.mark.parametrize("w", [8, 20, 40])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_far_logits_with_many_tiles(dtype, w):
    """Every logit equal and far (181 * 2^24 before the scale): plain means, to the bound of
    the sums, over all tiles again."""
    cache, table, lens = _long(dtype)
    batch = das.Batch(torch.tensor(lens, dtype=torch.int32, device=DEV), torch.as_tensor(table, device=DEV))
    codes = cache.k_pool.view(torch.uint8)
    codes.zero_()
    codes[..., key_bytes(64)[:, 0]] = 0x38  # 1
    q, kb, vb = _block(2, dtype, 13, w, 16, 16, 64)
    q.zero_()
    kb.zero_()
    q[..., 0], kb[..., 0] = 181 * 2.0 ** 24, 1.0
    out = das.attn_policy_q8(cache, batch, 0, 1, 1, q, kb, vb)
    host = HostCache(cache)
    for b in (0, 12):
        ref, _, a, _ = attention(host, table, lens, b, 0, 0, 0, q, kb, vb)
        tol = tolerance(dtype, ref, a, 0.0, lens[b] + w, 64)
        assert (np.abs(out[b].double().cpu().numpy() - ref) <= tol).all(), b
