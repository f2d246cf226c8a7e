"""Attention over the 8-bit cache at the ends of its types' ranges, against the 64-bit
oracle: block values far above and below the cache's."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2609_34538_amd import _lib as das
from q8_ref import HostCache, attention, random_cache, tolerance
from test_gpu_attn_q8 import _block

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32

# dtype, dh, group, w: every number of waves with different rows, one and two block tiles
SHAPES = [(BF16, 64, 1, 8), (BF16, 96, 1, 33), (BF16, 128, 2, 20), (BF16, 64, 8, 33), (BF16, 128, 4, 64),
          (F32, 64, 1, 8), (F32, 64, 2, 20), (F32, 96, 8, 33), (F32, 128, 2, 10)]
ids = lambda c: f"{str(c[0])[6:]}-dh{c[1]}-g{c[2]}-w{c[3]}"  # noqa: E731


def check(cache, batch, table, lens, q, kb, vb, unit=1.0):
    """Outputs within their bound, counted in units of `unit`."""
    out = das.attn_policy_q8(cache, batch, 0, 1, 1, q, kb, vb, out=torch.full_like(q, float("nan")))
    host = HostCache(cache)
    for b in range(len(lens)):
        ref, _, a, size = attention(host, table, lens, b, 0, 0, 0, q, kb, vb)
        tol = tolerance(cache.dtype, ref / unit, a / unit, size, lens[b] + q.shape[1], q.shape[3])
        err = np.abs(out[b].double().cpu().numpy() - ref) / unit
        assert (err <= tol).all(), (b, lens[b], float((err / tol).max()))
    return out


@pytest.mark.parametrize("lens", [[0, 0], [0, 40], [4000, 700]], ids=["none", "one-chunk", "chunks"])
@pytest.mark.parametrize("shape", SHAPES, ids=ids)
@pytest.mark.parametrize("e", [-100, 39, 40, 55, 60, 100, 110])
def test_block_values_of_any_size(e, shape, lens):
    """The same bound as for values of size 1, relative to the largest term of the sum."""
    dtype, dh, G, w = shape
    cache, batch, table = random_cache(7, dtype, 2, 2, dh, lens)
    q, kb, vb = _block(11, dtype, 2, w, 2 * G, 2, dh)
    check(cache, batch, table, lens, q, kb, vb * 2.0 ** e, 2.0 ** e if e > 0 or max(lens) == 0 else 1.0)


@pytest.mark.parametrize("shape", SHAPES, ids=ids)
def test_large_block_values_reach_only_the_rows_that_see_them(shape):
    dtype, dh, G, w = shape
    lens = [1500, 0]
    cache, batch, table = random_cache(7, dtype, 2, 2, dh, lens)
    q, kb, vb = _block(11, dtype, 2, w, 2 * G, 2, dh)
    clean = das.attn_policy_q8(cache, batch, 0, 1, 1, q, kb, vb)
    vb[:, 5], vb[:, w - 1, :, 3] = 2.0 ** 100, -2.0 ** 90
    out = check(cache, batch, table, lens, q, kb, vb)
    assert torch.equal(out[:, :5], clean[:, :5])
    assert bool((out[:, 5:].float() > 2.0 ** 60).all())
