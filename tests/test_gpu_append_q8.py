"""The commit into the 8-bit cache, byte for byte against a 64-bit reference of its
definition: everything it shall write, and nothing else."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2609_34538_amd import _lib as das
from q8_ref import HostCache, random_cache

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def _new(seed, cache, B, w, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    L, hkv, dh = cache.num_layers, cache.num_kv_heads, cache.head_dim
    return [(torch.randn((n, L, B, w, hkv, dh), generator=g, device=DEV) * scale).to(cache.dtype)
            for n in (cache.k_pool.shape[0], cache.v_pool.shape[0])]


def _assert_same(cache, host):
    got = HostCache(cache)
    for s in "kv":
        assert np.array_equal(got.exp[s], host.exp[s]), f"{s} exponents"
        a, b = got.pool[s], host.pool[s]
        nan = (a & 127 == 127) & (b & 127 == 127)  # either sign of NaN
        assert (nan | (a == b)).all(), f"{s} codes"


def _run(cache, batch, table, lens, k_new, v_new, num):
    host = HostCache(cache)
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    host.commit(table, lens, f(k_new), f(v_new), num)
    len_out = torch.full((len(lens),), -9, dtype=torch.int32, device=DEV)
    das.kv_append_q8(cache, batch, k_new, v_new,
                     torch.tensor(num, dtype=torch.int32, device=DEV), len_out)
    _assert_same(cache, host)
    assert len_out.tolist() == [s + n for s, n in zip(lens, num)]
    assert int(batch.dev_error) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dh", [64, 96, 128])
@pytest.mark.parametrize("w,lens,num", [
    (1, [0, 7, 8, 63, 64, 5], [1, 1, 1, 1, 1, 0]),
    (8, [0, 3, 60, 64, 121], [8, 8, 8, 5, 2]),
    (64, [0, 1, 63, 100], [64, 64, 64, 37]),
    (13, [50, 8], [13, 0]),
])
def test_bytes(dtype, dh, w, lens, num):
    cache, batch, table = random_cache(3, dtype, len(lens), 3, dh, lens, spare=64, layers=2, nk=2,
                                       garbage=False)
    _run(cache, batch, table, lens, *_new(5, cache, len(lens), w), num)


@pytest.mark.parametrize("scale", [2.0 ** -70, 2.0 ** -20, 0.01, 300.0, 2.0 ** 40, 2.0 ** 120])
def test_scales(scale):
    """New tokens far larger and far smaller than what their groups hold."""
    lens, num = [4, 8, 61], [9, 3, 5]
    cache, batch, table = random_cache(3, F32, 3, 2, 64, lens, spare=64, garbage=False, spread=3)
    _run(cache, batch, table, lens, *_new(5, cache, 3, 9, scale), num)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_special_values(dtype):
    """Zeros of both signs, ties, the border of the exponent, subnormal codes, the largest
    and smallest numbers, infinities and NaN."""
    lens, num = [0, 5], [16, 16]
    cache, batch, table = random_cache(3, dtype, 2, 2, 64, lens, spare=64, garbage=False)
    k_new, v_new = _new(1, cache, 2, 16)
    odd = [0.0, -0.0, 448.0, -448.0, 449.0, 17.0, 19.0, 2.0 ** -9, 3 * 2.0 ** -10, 2.0 ** -10, -1e-30,
           float("inf"), -float("inf"), float("nan"), torch.finfo(dtype).max, -torch.finfo(dtype).max,
           torch.finfo(dtype).tiny, 1.0625, 1.1875]
    for t in (k_new, v_new):
        flat = t.view(-1)
        for i, x in enumerate(odd):
            flat[137 * i + 5] = x
        t[:, :, :, 8:] = 0.0  # groups of zeros
        t[:, :, 0, 3] = 0.0
    _run(cache, batch, table, lens, k_new, v_new, num)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_token_by_token(dtype):
    """Single tokens whose sizes rise and fall, one commit after the other."""
    cache, batch, table = random_cache(3, dtype, 1, 2, 96, [0], spare=40, garbage=False)
    for s in range(20):
        batch = das.Batch(torch.tensor([s], dtype=torch.int32, device=DEV), batch.block_table,
                          batch.dev_error)
        _run(cache, batch, table, [s], *_new(s, cache, 1, 1, 2.0 ** (s * 7 % 11 - 5)), [1])


def test_bad_counts_and_pages_are_reported_and_skipped():
    lens, num = [0, 10, 30, 120, 70], [9, -1, 3, 20, 2]
    cache, batch, table = random_cache(3, BF16, 5, 1, 64, [0, 10, 30, 120, 70], spare=8, garbage=False)
    bad = table.copy()
    bad[4, 1] = cache.num_pages + 3
    batch = das.Batch(batch.prefix_len, torch.as_tensor(bad, device=DEV), batch.dev_error)
    k_new, v_new = _new(5, cache, 5, 8)
    host = HostCache(cache)
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    host.commit(bad, lens, f(k_new), f(v_new), [0, 0, 3, 0, 2])  # 9 > w, -1, and 140 > 2 pages
    len_out = torch.empty(5, dtype=torch.int32, device=DEV)
    das.kv_append_q8(cache, batch, k_new, v_new, torch.tensor(num, dtype=torch.int32, device=DEV), len_out)
    _assert_same(cache, host)
    assert len_out.tolist() == [0, 10, 33, 120, 72]
    assert int(batch.dev_error) == das.DEVERR_COMMIT | das.DEVERR_PAGE


def test_graph_replays_match_eager():
    lens, num = [3, 64], [8, 5]
    cache, batch, table = random_cache(3, BF16, 2, 2, 96, lens, spare=64, garbage=False)
    k_new, v_new = _new(5, cache, 2, 8)
    n = torch.tensor(num, dtype=torch.int32, device=DEV)
    state = [cache.k_pool, cache.v_pool, cache.k_exp, cache.v_exp]
    before = [t.clone() for t in state]
    das.kv_append_q8(cache, batch, k_new, v_new, n)
    want = [t.clone() for t in state]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        das.kv_append_q8(cache, batch, k_new, v_new, n)
    for _ in range(4):
        for t, b in zip(state, before):
            t.copy_(b)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t.view(torch.uint8), w.view(torch.uint8)) for t, w in zip(state, want))
