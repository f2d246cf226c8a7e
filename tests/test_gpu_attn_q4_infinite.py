"""fp32 and bf16 attention over the 4-bit cache with infinities and NaN of any bits among the
block keys that a row sees."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2609_34538_amd import _lib as das
from q4_ref import random_cache
from test_gpu_attn_q4 import BF16, DEV, F32, _block

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dh", [64, 96, 128])
@pytest.mark.parametrize("w,at", [(9, 2), (20, 2), (40, 35), (64, 40)])
def test_keys_of_minus_infinity_take_no_part(dtype, dh, w, at):
    """A logit of -infinity is a weight of 0, as a far one is; rows that take it times 0 and
    those of a logit of +infinity are NaN, and rows before it are as they were."""
    cache, batch, _ = random_cache(8, dtype, 1, 2, dh, [100])
    q, kb, vb = _block(3, dtype, 1, w, 4, 2, dh)
    q = torch.round(q * 4) / 4  # no bits below bf16's
    q[0, :, :2, 7] = q[0, :, :2, 7].abs() + 0.25
    q[0, at + 3, 0, 7] = 0.0
    clean = das.attn_policy_q4(cache, batch, 0, 1, 1, q, kb, vb)
    kb[0, at, 0, 7] = -2.0 ** 100
    want = das.attn_policy_q4(cache, batch, 0, 1, 1, q, kb, vb)
    assert torch.isfinite(want).all() and torch.equal(want[:, :at], clean[:, :at])
    kb[0, at, 0, 7] = -float("inf")
    lse = torch.empty((1, 4, w), device=DEV)
    out = das.attn_policy_q4(cache, batch, 0, 1, 1, q, kb, vb, lse=lse)
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[0, at + 3, 0] = True
    assert torch.isnan(out[hit]).all() and torch.equal(out[~hit], want[~hit])
    assert torch.equal(torch.isfinite(lse[0].T), ~hit[0, :, :, 0])
    kb[0, at, 0, 7] = float("inf")
    out = das.attn_policy_q4(cache, batch, 0, 1, 1, q, kb, vb)
    assert torch.isnan(out[0, at:, :2]).all() and torch.isfinite(out[0, :at]).all()
    assert torch.isfinite(out[0, :, 2:]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("w", [9, 40])
@pytest.mark.parametrize("negative", [False, True])
def test_a_nan_key_of_any_bits_is_seen(dtype, w, negative):
    """The NaN whose upper bits alone would be an infinity among them."""
    cache, batch, _ = random_cache(8, dtype, 1, 2, 64, [100])
    q, kb, vb = _block(3, dtype, 1, w, 2, 2, 64)
    clean = das.attn_policy_q4(cache, batch, 0, 1, 1, q, kb, vb)
    bits = 0x7f800001 if dtype == F32 else 0x7f81
    word = np.array([bits | (0x80000000 if dtype == F32 else 0x8000) * negative],
                    dtype=np.uint32 if dtype == F32 else np.uint16)
    kb[0, 4, 1, 9:10] = torch.as_tensor(word.view(np.int32 if dtype == F32 else np.int16)).view(dtype).to(DEV)
    out = das.attn_policy_q4(cache, batch, 0, 1, 1, q, kb, vb)
    assert torch.isnan(out[0, 4:, 1]).all()
    out[0, 4:, 1] = clean[0, 4:, 1]
    assert torch.equal(out, clean)
