"""The commit into the 4-bit cache, byte for byte against a 64-bit reference of its
definition, everything it shall write and nothing else; and the way back."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2609_34538_amd import _lib as das
from q4_ref import NAN_BYTE, PAGE, HostCache, random_cache

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
I32 = dict(dtype=torch.int32, device=DEV)


def _rows(cache, B, w, value=0.0):
    L, hkv, dh = cache.num_layers, cache.num_kv_heads, cache.head_dim
    return [torch.full((n, L, B, w, hkv, dh), value, dtype=cache.dtype, device=DEV)
            for n in (cache.k_pool.shape[0], cache.v_pool.shape[0])]


def _new(seed, cache, B, w, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return [(torch.randn(x.shape, generator=g, device=DEV) * scale).to(cache.dtype)
            for x in _rows(cache, B, w)]


def _assert_same(cache, host):
    got = HostCache(cache)
    for s in "kv":
        assert np.array_equal(got.exp[s], host.exp[s]), f"{s} exponents"
        assert np.array_equal(got.pool[s], host.pool[s]), f"{s} codes"


def _f(t):
    return t.double().cpu().numpy()


def _run(cache, batch, table, lens, k_new, v_new, num):
    host = HostCache(cache)
    host.commit(table, lens, _f(k_new), _f(v_new), num)
    len_out = torch.full((len(lens),), -9, **I32)
    das.kv_append_q4(cache, batch, k_new, v_new, torch.tensor(num, **I32), len_out)
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
    cache, batch, table = random_cache(3, dtype, len(lens), 3, dh, lens, spare=64, layers=2, nk=2)
    _run(cache, batch, table, lens, *_new(5, cache, len(lens), w), num)


@pytest.mark.parametrize("scale", [2.0 ** -135, 2.0 ** -122, 2.0 ** -60, 0.01, 300.0, 2.0 ** 60, 2.0 ** 124])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_sizes(dtype, scale):
    """Values from below the smallest scale to the largest."""
    lens = [10, 64]
    cache, batch, table = random_cache(3, dtype, 2, 2, 64, lens, spare=64)
    _run(cache, batch, table, lens, *_new(5, cache, 2, 9, scale), [9, 4])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_borders(dtype):
    """Values on and beside every border of the codes, under scales whose choice is on a
    border too (a block's largest 6.9, 7, 7.1, 14), zeros and the largest numbers."""
    lens = [3]
    cache, batch, table = random_cache(3, dtype, 1, 1, 64, lens, spare=64)
    k, v = _rows(cache, 1, 24)
    border = torch.tensor([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6], dtype=torch.float64)
    step = 2.0 ** -8 if dtype == BF16 else 2.0 ** -23
    x = torch.cat([border, border * (1 + step)])  # 30 values
    fmax = torch.finfo(dtype).max
    for i, top in enumerate([6.9, 7.0, 7.1, 14.0, 3.5, 0.0, -7.0, 6.0]):
        for j, scale in enumerate([1.0, 2.0 ** -30, -2.0 ** 90]):
            row = torch.zeros(64, dtype=torch.float64)
            row[:30], row[31], row[32] = x * scale, top * scale, 1e-3 * scale
            k[0, 0, 0, 3 * i + j, 0] = row.to(dtype)
    v.copy_(k.flip(-1))
    v[0, 0, 0, 5, 0, 3], v[0, 0, 0, 6, 0, 4], k[0, 0, 0, 7] = fmax, -fmax, 0.0
    _run(cache, batch, table, lens, k, v, [24])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_what_is_not_finite_makes_its_block_nan(dtype):
    lens = [3]
    cache, batch, table = random_cache(3, dtype, 1, 2, 96, lens, spare=64)
    k, v = _new(5, cache, 1, 6)
    k[0, 0, 0, 1, 0, 33], k[0, 0, 0, 2, 1, 0] = float("inf"), float("nan")
    v[0, 0, 0, 4, 0, 95], v[0, 0, 0, 5, 1, 31] = -float("inf"), float("nan")
    before = HostCache(cache)
    das.kv_append_q4(cache, batch, k, v, torch.tensor([6], **I32))
    host = HostCache(cache)
    for side, x in (("k", k), ("v", v)):
        got = host.rows(side, 0, 0, table[0], 9)[3:]                     # [6, 2, 96]
        finite = torch.isfinite(x[0, 0, 0]).view(6, 2, 3, 32).all(-1).cpu().numpy()
        assert np.array_equal(np.isfinite(got).reshape(6, 2, 3, 32).all(-1), finite)
        assert np.isnan(got.reshape(6, 2, 3, 32)[~finite]).all() and (~finite).sum() == 2
        # the others are as if they were alone, and earlier tokens as they were
        clean = before.rows(side, 0, 0, table[0], 3)
        assert np.array_equal(host.rows(side, 0, 0, table[0], 3), clean)
        before.write(side, 0, 0, table[0][0], 20, np.where(np.isfinite(_f(x[0, 0, 0, 0])), _f(x[0, 0, 0, 0]), 0))


def test_tokens_one_by_one_or_together():
    """The same bytes whatever tokens are committed together."""
    caches = [random_cache(3, BF16, 1, 2, 96, [5], spare=128) for _ in range(2)]
    k, v = _new(5, caches[0][0], 1, 30)
    cache, batch, _ = caches[0]
    das.kv_append_q4(cache, batch, k, v, torch.tensor([30], **I32))
    cache2, batch2, _ = caches[1]
    at = 0
    for n in (1, 2, 7, 8, 12):
        das.kv_append_q4(cache2, batch2, k[:, :, :, at:at + n].contiguous(), v[:, :, :, at:at + n].contiguous(),
                         torch.tensor([n], **I32), nxt := torch.empty(1, **I32))
        batch2 = das.Batch(nxt, batch2.block_table)
        at += n
    for a, b in zip((cache.k_pool, cache.v_pool, cache.k_exp, cache.v_exp),
                    (cache2.k_pool, cache2.v_pool, cache2.k_exp, cache2.v_exp)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_bad_counts_and_pages(dtype):
    """Counts out of range leave the sequence alone, unreadable pages their positions."""
    lens = [60, 10, 20, 100, 5]
    cache, batch, table = random_cache(3, dtype, 5, 2, 64, lens, spare=64)
    bad = table.copy()
    bad[0, 1] = cache.num_pages  # positions 64.. of sequence 0
    batch = das.Batch(batch.prefix_len, torch.as_tensor(bad, device=DEV), batch.dev_error)
    k, v = _new(5, cache, 5, 16)
    num = [16, -1, 17, 2 ** 31 - 1, 3]
    host = HostCache(cache)
    host.commit(bad, lens, _f(k), _f(v), [16, 0, 0, 0, 3])
    out = torch.full((5,), -9, **I32)
    das.kv_append_q4(cache, batch, k, v, torch.tensor(num, **I32), out)
    _assert_same(cache, host)
    assert out.tolist() == [76, 10, 20, 100, 8]
    assert int(batch.dev_error) == das.DEVERR_PAGE | das.DEVERR_COMMIT


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dh", [64, 96, 128])
@pytest.mark.parametrize("w,first,num", [
    (1, [0, 70, 299], [1, 0, 1]),
    (9, [60, 7, 291], [9, 8, 9]),
    (300, [0, 3, 100], [300, 77, 200]),
])
def test_read_back(dtype, dh, w, first, num):
    """Elements as they stand for, rows past the count left alone."""
    lens = [300, 80, 300]
    cache, batch, table = random_cache(4, dtype, 3, 3, dh, lens, layers=2, nk=2, spread=2)
    host = HostCache(cache)
    got = _rows(cache, 3, w, 7.0)
    das.kv_read_q4(cache, batch, torch.tensor(first, **I32), torch.tensor(num, **I32), *got)
    for side, x in zip("kv", got):
        for p in range(x.shape[0]):
            for la in range(2):
                for b in range(3):
                    want = host.rows(side, p, la, table[b], lens[b])[first[b]:first[b] + num[b]]
                    assert np.array_equal(_f(x[p, la, b, :num[b]]), want), (side, p, la, b)
                    assert (x[p, la, b, num[b]:] == 7).all()
    assert int(batch.dev_error) == 0


def test_read_refuses_positions_outside_the_prefix():
    lens = [100, 100, 100, 100, 100]
    cache, batch, table = random_cache(4, BF16, 5, 2, 64, lens)
    bad = table.copy()
    bad[4, 1] = -1
    batch = das.Batch(batch.prefix_len, torch.as_tensor(bad, device=DEV), batch.dev_error)
    got = _rows(cache, 5, 50, 7.0)
    first, num = [60, -1, 10, 0, 50], [41, 5, 51, -2, 50]
    das.kv_read_q4(cache, batch, torch.tensor(first, **I32), torch.tensor(num, **I32), *got)
    host = HostCache(cache)
    for side, x in zip("kv", got):
        assert (x[:, :, :4] == 7).all()
        want = host.rows(side, 0, 0, table[4], 64)[50:]
        assert np.array_equal(_f(x[0, 0, 4, :14]), want) and (x[0, 0, 4, 14:] == 7).all()
    assert int(batch.dev_error) == das.DEVERR_PREFIX | das.DEVERR_PAGE


def test_nan_blocks_read_as_nan():
    cache, batch, table = random_cache(4, BF16, 1, 1, 64, [70], garbage=False)
    cache.k_exp[0, 0, 0, int(table[0, 0]), 0, 1] = NAN_BYTE  # token 0, dims 32..63
    got = _rows(cache, 1, 70)
    das.kv_read_q4(cache, batch, torch.zeros(1, **I32), torch.tensor([70], **I32), *got)
    assert torch.isnan(got[0][0, 0, 0, 0, 0, 32:]).all() and torch.isfinite(got[0][0, 0, 0, 0, 0, :32]).all()
    assert torch.isfinite(got[0][0, 0, 0, 1:]).all() and torch.isfinite(got[1]).all()


def test_what_is_read_commits_to_the_same_elements():
    """A prefix moved to another 4-bit cache; elements of a block whose largest is 0.5 or 1
    of a scale come back under a smaller one."""
    lens = [130]
    cache, batch, table = random_cache(4, BF16, 1, 3, 96, lens)
    got = _rows(cache, 1, 64)
    other, batch2, table2 = random_cache(9, BF16, 1, 3, 96, [0], spare=200)
    at = 0
    while at < 130:
        n = min(64, 130 - at)
        das.kv_read_q4(cache, batch, torch.tensor([at], **I32), torch.tensor([n], **I32), *got)
        nxt = torch.empty(1, **I32)
        das.kv_append_q4(other, batch2, *got, torch.tensor([n], **I32), nxt)
        batch2 = das.Batch(nxt, batch2.block_table)
        at += n
    a, b = HostCache(cache), HostCache(other)
    for s in "kv":
        assert np.array_equal(a.rows(s, 0, 0, table[0], 130), b.rows(s, 0, 0, table2[0], 130))


def test_offsets_past_32_bits():
    """A pool of over 4 GiB: its last pages."""
    hkv, dh, pages = 64, 128, 17000
    assert hkv * pages * 32 * dh > 1 << 32
    cache = das.Quant4Cache.empty(1, hkv, pages, dh, 1, {1: 0}, {1: 0})
    table = torch.tensor([[pages - 1, 0]], **I32)
    batch = das.Batch(torch.tensor([60], **I32), table)
    k, v = _new(5, cache, 1, 8)
    new_len = torch.empty(1, **I32)
    das.kv_append_q4(cache, batch, k, v, torch.tensor([8], **I32), new_len)
    got = _rows(cache, 1, 8)
    das.kv_read_q4(cache, das.Batch(new_len, table), torch.tensor([60], **I32), torch.tensor([8], **I32), *got)
    for x, y in zip(got, (k, v)):
        z = _f(y)[0, 0, 0].reshape(8, hkv, 4, 32)
        # within half the distance of the largest codes, of scales up to 2/3.5 of the largest
        assert (np.abs(_f(x)[0, 0, 0].reshape(z.shape) - z) <= np.abs(z).max(-1, keepdims=True) / 3.5 + 1e-30).all()
    assert int((cache.k_pool[0, 0, :, 1:pages - 1] != 0).sum()) == 0
    q = torch.randn((1, 1, hkv, dh), device=DEV).to(BF16)
    kb = torch.zeros((1, 1, hkv, dh), device=DEV, dtype=BF16)
    out = das.attn_policy_q4(cache, das.Batch(new_len, table), 0, 1, 1, q, kb, kb)
    ks, vs = (x[0, 0, 0].double() for x in got)                          # [8, hkv, dh]
    x = torch.cat([torch.zeros((60, hkv), device=DEV, dtype=torch.float64), (q[0, 0].double() * ks).sum(-1)
                   / dh ** 0.5, torch.zeros((1, hkv), device=DEV, dtype=torch.float64)])
    ref = (torch.softmax(x, 0)[60:68, :, None] * vs).sum(0)
    assert (out[0, 0].double() - ref).abs().max() < 0.02
