"""Attention over the 8-bit cache at the ends of its types' ranges, against the 64-bit
oracle: block values far above and below the cache's, and logits of any size."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2609_34538_amd import _lib as das
from q8_ref import HostCache, attention, key_bytes, random_cache, tolerance
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
        n = lens[b] + q.shape[1]
        tol = tolerance(cache.dtype, ref / unit, a / unit, size, n, q.shape[3])
        # under the smallest normal: half a step of bf16; half steps of fp32 in each sum, whose
        # weights add up to 2^-6 or more
        tol += (2.0 ** -134 if cache.dtype == BF16 else (n + 2) * 2.0 ** -144) / unit
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


def _alone(cache, e, sign, B, w, hq, dh):
    """Keys of the cache and the block, and queries, that give every position the logit
    sign * 181 / 128 * 2^e before the scale, exactly: all in dimension 0. Returns (q, k_blk)."""
    c = max(min(e // 2, 110), -60)
    codes = cache.k_pool.view(torch.uint8)
    codes.zero_()
    codes[..., key_bytes(dh)[:, 0]] = 0x38  # 1
    cache.k_exp.copy_(torch.where(cache.k_exp == 255, cache.k_exp, torch.full_like(cache.k_exp, 127 + c)))
    q = torch.zeros((B, w, hq, dh), dtype=cache.dtype, device=DEV)
    kb = torch.zeros((B, w, cache.num_kv_heads, dh), dtype=cache.dtype, device=DEV)
    q[..., 0], kb[..., 0] = sign * 181 / 128 * 2.0 ** (e - c), 2.0 ** c
    return q, kb


@pytest.mark.parametrize("lens", [[0, 40], [4000, 700]], ids=["one-chunk", "chunks"])
@pytest.mark.parametrize("shape", SHAPES, ids=ids)
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("e", [3, 20, 24, 27, 31, 60, 104, 120])
def test_logits_of_any_size(e, sign, shape, lens):
    """Equal logits are averaged, and twice the logit from block position 3 on takes all or
    leaves all, whatever their size. The logits are exact, so they add nothing to the bound
    but the fp32 steps of 2^e in the logarithm."""
    dtype, dh, G, w = shape
    cache, batch, table = random_cache(7, dtype, 2, 2, dh, lens)
    _, _, vb = _block(11, dtype, 2, w, 2 * G, 2, dh)
    q, kb = _alone(cache, e, sign, 2, w, 2 * G, dh)
    host = HostCache(cache)
    for twice in (False, True):
        if twice:
            kb[:, 3:] *= 2
        lse = torch.full((2, 2 * G, w), float("nan"), device=DEV)
        out = das.attn_policy_q8(cache, batch, 0, 1, 1, q, kb, vb, lse=lse)
        for b in range(2):
            ref, rl, a, _ = attention(host, table, lens, b, 0, 0, 0, q, kb, vb)
            tol = tolerance(dtype, ref, a, 0.0, lens[b] + w, dh)
            err = np.abs(out[b].double().cpu().numpy() - ref)
            assert (err <= tol).all(), (b, twice, float((err / tol).max()))
            lt = 2 * (lens[b] + 80) * 2.0 ** -24 + 2.0 ** -21 * np.abs(rl)
            assert (np.abs(lse[b].double().cpu().numpy() - rl) <= lt).all(), (b, twice)


@pytest.mark.parametrize("shape", SHAPES, ids=ids)
def test_large_logits_and_block_values(shape):
    """Rows that reach far logits step by step, with values that are added at the end."""
    dtype, dh, G, w = shape
    lens = [500, 0]
    cache, batch, table = random_cache(7, dtype, 2, 2, dh, lens)
    _, _, vb = _block(11, dtype, 2, w, 2 * G, 2, dh)
    vb *= 2.0 ** 60
    q, kb = _alone(cache, 10, 1, 2, w, 2 * G, dh)
    kb[..., 0] *= 2.0 ** (torch.arange(w, device=DEV) * 3 % 32)[None, :, None]
    host = HostCache(cache)
    out = das.attn_policy_q8(cache, batch, 0, 1, 1, q, kb, vb)
    for b in range(2):
        ref, _, a, _ = attention(host, table, lens, b, 0, 0, 0, q, kb, vb)
        tol = tolerance(dtype, ref, a, 0.0, lens[b] + w, dh)
        assert (np.abs(out[b].double().cpu().numpy() - ref) <= tol).all(), b


@pytest.mark.parametrize("shape", SHAPES, ids=ids)
def test_values_up_to_the_largest(shape):
    """Two prefix values of 1.5 * 2^126 whose logits pass those that a wave has met before by
    a few binary orders: their sum is 3/4 of the largest fp32. Weights 2^3.5 or more against at
    most 190 of 1: the two have a tenth of the sum, the output is over 2^123."""
    dtype, dh, G, w = shape
    lens = [128, 128]
    cache, batch, table = random_cache(7, dtype, 2, 2, dh, lens)
    q = torch.zeros((2, w, 2 * G, dh), dtype=dtype, device=DEV)
    kb = torch.zeros((2, w, 2, dh), dtype=dtype, device=DEV)
    q[..., 0] = 8
    for pool in (cache.k_pool, cache.v_pool):
        pool.view(torch.uint8).zero_()
    cache.k_exp.fill_(127)
    cache.v_exp.fill_(63)
    tiles = (2 - (w + 31) // 32, 4 - (w + 31) // 32)
    for b in range(2):
        for t in (32 * i + 5 for i in tiles):
            page, group, j = int(table[b, t // 64]), t % 64 // 8, t % 8
            cache.k_pool.view(torch.uint8)[0, 0, :, page, group, int(key_bytes(dh)[j, 0])] = 0x46  # 3.5
            cache.v_pool.view(torch.uint8)[0, 0, :, page, group, :, j] = 0x74  # 192
            cache.v_exp[0, 0, page, :, group] = 119 + 127
    out = check(cache, batch, table, lens, q, kb, torch.ones_like(kb), 2.0 ** 126)
    assert bool((out.float() > 2.0 ** 123).all())


@pytest.mark.parametrize("block", ["zero", "tiny", "alike"])
@pytest.mark.parametrize("lens", [[40, 1], [4000, 700]], ids=["one-chunk", "chunks"])
@pytest.mark.parametrize("shape", SHAPES, ids=ids)
@pytest.mark.parametrize("byte", [1, 8, 20, 38, 62, 247])
def test_scales_of_any_size(byte, shape, lens, block):
    """A cache whose values all have one exponent byte, down to the smallest, and one past
    what the commit gives; block values of 0, of 2^-100, and of the cache's size."""
    dtype, dh, G, w = shape
    cache, batch, table = random_cache(7, dtype, 2, 2, dh, lens)
    cache.v_exp.copy_(torch.where(cache.v_exp == 255, cache.v_exp, torch.full_like(cache.v_exp, byte)))
    if byte > 246:  # codes under 1: thousands of values whose sum fits fp32
        codes = cache.v_pool.view(torch.uint8)
        codes.copy_(torch.where(codes & 0x7f == 0x7f, codes, codes & 0x9f))
    q, kb, vb = _block(11, dtype, 2, w, 2 * G, 2, dh)
    vb *= {"zero": 0.0, "tiny": 2.0 ** -100, "alike": 2.0 ** (byte - 127)}[block]
    check(cache, batch, table, lens, q, kb, vb, max(2.0 ** (byte - 127), float(vb.abs().max())))
