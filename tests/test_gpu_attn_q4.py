"""Attention over the 4-bit cache against the 64-bit oracle on the decoded cache: types,
head dims, head layouts, widths, lengths around groups, tiles and pages, unlike exponents,
NaN in every place that holds no token, unreadable pages, streams and graphs."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2609_34538_amd import _lib as das
from q4_ref import HostCache, attention, logit_error, random_cache, tolerance

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def _block(seed, dtype, B, w, hq, hkv, dh, gain=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda h: torch.randn((B, w, h, dh), generator=g, device=DEV)  # noqa: E731
    return (r(hq) * gain).to(dtype), r(hkv).to(dtype), r(hkv).to(dtype)


def _check(cache, batch, table, lens, q, kb, vb, out, lse, seqs=None, layer=0, kappa=1, nu=1):
    host = HostCache(cache)
    for b in range(len(lens)) if seqs is None else seqs:
        ref, rl, a, size = attention(host, table, lens, b, layer, kappa - 1, nu - 1, q, kb, vb)
        got = out[b].double().cpu().numpy()
        tol = tolerance(cache.dtype, ref, a, size, lens[b] + q.shape[1], q.shape[3])
        err = np.abs(got - ref)
        assert (err <= tol).all(), (b, lens[b], float((err / tol).max()))
        # the logit's and the sum's share of the bound, in the logarithm, and its fp32 steps
        lt = (2 * logit_error(cache.dtype, size, q.shape[3]) + 2 * (lens[b] + 80) * 2.0 ** -24
              + 2.0 ** -22 * np.abs(rl))
        le = np.abs(lse[b].double().cpu().numpy() - rl)
        assert (le <= lt).all(), (b, lens[b], float((le / lt).max()))


def _run(cache, batch, q, kb, vb, layer=0, kappa=1, nu=1):
    lse = torch.full((q.shape[0], q.shape[2], q.shape[1]), float("nan"), device=DEV)
    out = das.attn_policy_q4(cache, batch, layer, kappa, nu, q, kb, vb,
                             out=torch.full_like(q, float("nan")), lse=lse)
    return out, lse


CASES = [  # dtype, dh, hkv, group, w, lens, spread
    (BF16, 64, 2, 1, 1, [0, 1, 7, 8, 9], 0),
    (BF16, 96, 3, 1, 4, [31, 32, 33, 63, 64, 65, 127, 128, 129], 1),
    (BF16, 128, 2, 4, 8, [300, 0, 95], 2),
    (BF16, 128, 1, 8, 64, [1000, 77], 0),
    (BF16, 64, 4, 7, 5, [640, 513], 1),
    (BF16, 96, 2, 2, 33, [200, 1], 1),
    (BF16, 96, 55, 1, 16, [700], 0),
    (BF16, 96, 5, 1, 31, [39, 450], 1),
    (BF16, 64, 1, 1, 64, [4097], 1),
    (BF16, 64, 2, 1, 40, [70, 0], 1),
    (BF16, 128, 2, 1, 1, [9000, 3], 0),
    (BF16, 128, 3, 1, 24, [130, 1999], 1),
    (BF16, 128, 2, 2, 23, [61, 100], 1),
    (F32, 64, 4, 1, 4, [256, 0, 1], 0),
    (F32, 96, 2, 1, 17, [65, 500], 2),
    (F32, 96, 1, 8, 11, [129], 1),
    (F32, 128, 2, 4, 32, [333, 64], 1),
    (F32, 128, 1, 1, 1, [2500, 8], 0),
    (F32, 64, 1, 8, 64, [50], 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{str(c[0])[6:]}-dh{c[1]}-h{c[2]}x{c[3]}-w{c[4]}-{c[5][0]}")
def test_matches_the_oracle(case):
    dtype, dh, hkv, G, w, lens, spread = case
    B = len(lens)
    cache, batch, table = random_cache(7, dtype, B, hkv, dh, lens, spread=spread)
    q, kb, vb = _block(11, dtype, B, w, hkv * G, hkv, dh)
    out, lse = _run(cache, batch, q, kb, vb)
    _check(cache, batch, table, lens, q, kb, vb, out, lse)
    assert int(batch.dev_error) == 0


RAGGED = [  # dtype, dh, hkv, group, w, lens: many units of unlike lengths
    (BF16, 96, 55, 1, 16, [2000, 0, 1300, 4100, 64, 1]),
    (BF16, 64, 40, 1, 20, [1500, 3000, 33]),
    (BF16, 128, 16, 4, 1, [1, 4099, 700, 2048]),
    (BF16, 128, 16, 4, 33, [3001, 100]),
    (BF16, 96, 24, 8, 7, [500, 4000, 0]),
    (BF16, 64, 16, 8, 40, [4000, 1111]),
    (F32, 96, 30, 1, 9, [3500, 0, 129]),
    (F32, 64, 40, 2, 12, [2600, 1000]),
    (F32, 128, 16, 4, 11, [4000, 555]),
    (F32, 128, 16, 7, 64, [3900]),
]


@pytest.mark.parametrize("case", RAGGED, ids=lambda c: f"{str(c[0])[6:]}-dh{c[1]}-h{c[2]}x{c[3]}-w{c[4]}-{c[5][0]}")
def test_ragged_batches_match_the_oracle(case):
    """Units of one chunk, of several and of the block only; a wider table; equal bits
    again; and an unreadable page among them."""
    dtype, dh, hkv, G, w, lens = case
    B = len(lens)
    cache, batch, table = random_cache(7, dtype, B, hkv, dh, lens, spread=1)
    wide = torch.nn.functional.pad(batch.block_table, (0, 5), value=-1).contiguous()
    batch = das.Batch(batch.prefix_len, wide, batch.dev_error)
    q, kb, vb = _block(11, dtype, B, w, hkv * G, hkv, dh)
    out, lse = _run(cache, batch, q, kb, vb)
    _check(cache, batch, table, lens, q, kb, vb, out, lse)
    assert int(batch.dev_error) == 0
    assert torch.equal(out, das.attn_policy_q4(cache, batch, 0, 1, 1, q, kb, vb))
    b = int(np.argmax(lens))
    wide[b, 2] = -7
    keep = np.arange(lens[b]) // 64 != 2
    out = das.attn_policy_q4(cache, batch, 0, 1, 1, q, kb, vb)
    assert int(batch.dev_error) == das.DEVERR_PAGE
    ref, _, a, size = attention(HostCache(cache), table, lens, b, 0, 0, 0, q, kb, vb, keep=keep)
    tol = tolerance(dtype, ref, a, size, lens[b] + w, dh)
    assert (np.abs(out[b].double().cpu().numpy() - ref) <= tol).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dh", [64, 96, 128])
@pytest.mark.parametrize("group,w", [(1, 16), (1, 17), (2, 16), (3, 11), (1, 64), (5, 13), (8, 16), (8, 17)])
def test_rows_around_the_launch_shapes(dtype, dh, group, w):
    """16, 17, 32, 33, 64, 65, 128 and 136 query rows a KV head; chunks of one and several."""
    lens = [1500, 63, 0]
    cache, batch, table = random_cache(7, dtype, 3, 2, dh, lens, spread=1)
    q, kb, vb = _block(11, dtype, 3, w, 2 * group, 2, dh)
    out, lse = _run(cache, batch, q, kb, vb)
    _check(cache, batch, table, lens, q, kb, vb, out, lse)


@pytest.mark.parametrize("w", [4, 20, 32, 50])
def test_wide_heads_far_logits_and_late_values(w):
    """Head dim 128: infinities in block values reach who sees them, and rows whose logits are
    far give the value of the largest."""
    lens = [400]
    cache, batch, table = random_cache(9, BF16, 1, 2, 128, lens)
    q, kb, vb = _block(3, BF16, 1, w, 2, 2, 128)
    clean = das.attn_policy_q4(cache, batch, 0, 1, 1, q, kb, vb)
    vb[0, 3, 1, 100] = float("inf")
    out = das.attn_policy_q4(cache, batch, 0, 1, 1, q, kb, vb)
    assert torch.isinf(out[0, 3:, 1, 100]).all()
    out[0, 3:, 1, 100] = clean[0, 3:, 1, 100]
    assert torch.equal(out, clean)
    vb[0, 3, 1, 100] = 0
    cache.k_exp.copy_(torch.where(cache.k_exp == 255, 255, 127 + 30))
    kb.zero_()  # the largest logit is a cached token's, at 2^30 and more
    out = das.attn_policy_q4(cache, batch, 0, 1, 1, q, kb, vb)
    host = HostCache(cache)
    k, v = (host.rows(n, 0, 0, table[0], lens[0]) for n in ("k", "v"))
    for h in range(2):
        x = q[0, :, h].double().cpu().numpy() @ k[:, h].T / np.sqrt(128)
        top = np.sort(x, -1)[:, -2:]
        # fp32 sums of 128 exact products: 2^-17 of their sizes' sum at most
        err = 2.0 ** -16 * (np.abs(q[0, :, h].double().cpu().numpy()) @ np.abs(k[:, h]).T).max(-1) / np.sqrt(128)
        sure = top[:, 1] - top[:, 0] > 2 * err + 60
        assert sure.sum() > w // 2
        best = v[x.argmax(-1), h]
        got = out[0, :, h].double().cpu().numpy()
        # one probability of 1, what is under 2^-39 of the row's largest may be lost in a record,
        # whose elements have 11 bits, and a rounding to bf16
        tol = (2.0 ** -8 + 2.0 ** -11) * np.abs(best) + 2.0 ** -38 * np.abs(best).max(-1, keepdims=True)
        assert (np.abs(got - best) <= tol)[sure].all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_plane_layer_and_policy(dtype):
    """Keys of depth 2 and values of depth 3 at layer 1 are the ones that are read."""
    lens = [130, 40]
    cache, batch, table = random_cache(3, dtype, 2, 2, 64, lens, layers=2, nk=2, nv=3)
    q, kb, vb = _block(4, dtype, 2, 6, 4, 2, 64)
    out, lse = _run(cache, batch, q, kb, vb, 1, 2, 3)
    _check(cache, batch, table, lens, q, kb, vb, out, lse, layer=1, kappa=2, nu=3)


@pytest.mark.parametrize("dtype,w", [(BF16, 3), (BF16, 16), (F32, 4)])
def test_many_long_units(dtype, w):
    """More units than workgroups, over 64 pages to a wave or workgroup of one chunk (a
    second window of page ids)."""
    B, hkv, dh, S, pages = 70, 8, 64, 17000, 270
    g = torch.Generator(device=DEV).manual_seed(1)
    cache = das.Quant4Cache.empty(1, hkv, pages, dh, 1, {1: 0}, {1: 0}, dtype=dtype)
    for pool in (cache.k_pool, cache.v_pool):
        pool.copy_(torch.randint(0, 256, pool.shape, generator=g, device=DEV, dtype=torch.uint8))
    for exp in (cache.k_exp, cache.v_exp):
        exp.copy_(torch.randint(125, 127, exp.shape, generator=g, device=DEV, dtype=torch.uint8))
    n = -(-S // 64)
    table = np.stack([np.random.default_rng(b).permutation(pages)[:n] for b in range(B)]).astype(np.int32)
    lens = [S] * B
    batch = das.Batch(torch.full((B,), S, dtype=torch.int32, device=DEV),
                      torch.as_tensor(table, device=DEV))
    q, kb, vb = _block(2, dtype, B, w, 8 * hkv, hkv, dh)
    out, lse = _run(cache, batch, q, kb, vb)
    _check(cache, batch, table, lens, q, kb, vb, out, lse, seqs=[0, 69])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("w", [9, 40])
def test_unlike_exponents(dtype, w):
    """Scales of a unit's blocks over 2^-60 .. 2^60, and in one head over 2^-120 .. 2^-60."""
    lens = [257, 700]
    cache, batch, table = random_cache(5, dtype, 2, 2, 96, lens)
    rng = np.random.default_rng(0)
    e = rng.integers(67, 188, size=cache.v_exp.shape).astype(np.uint8)
    e[:, :, 1] = rng.integers(7, 68, size=e[:, :, 1].shape)
    cache.v_exp.copy_(torch.where(cache.v_exp == 255, cache.v_exp, torch.as_tensor(e, device=DEV)))
    q, kb, vb = _block(6, dtype, 2, w, 2, 2, 96)
    vb[:, :, 1] = 0  # what the tiny ones add up to shows
    out, lse = _run(cache, batch, q, kb, vb)
    host = HostCache(cache)
    for b in range(2):
        ref, _, a, size = attention(host, table, lens, b, 0, 0, 0, q, kb, vb)
        got = out[b].double().cpu().numpy()
        tol = tolerance(dtype, ref, a, size, lens[b] + w, 96)
        assert (np.abs(got - ref) <= tol).all(), float((np.abs(got - ref) / tol).max())
        assert np.abs(ref[:, 1]).max() < 2.0 ** -55 and np.abs(got[:, 1]).max() > 2.0 ** -70


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_block_values_of_any_size(dtype):
    """Block values near the largest number beside a cache of ordinary ones."""
    lens = [90]
    cache, batch, table = random_cache(5, dtype, 1, 2, 64, lens)
    q, kb, vb = _block(6, dtype, 1, 20, 2, 2, 64)
    vb[:, 3::5] *= 2.0 ** 120
    out, lse = _run(cache, batch, q, kb, vb)
    assert torch.isfinite(out).all()
    _check(cache, batch, table, lens, q, kb, vb, out, lse)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("w", [7, 48])
def test_large_logits(dtype, w):
    """Logits of some hundreds, whose softmax is one-hot nearly everywhere."""
    lens = [900, 65]
    cache, batch, table = random_cache(9, dtype, 2, 2, 128, lens, k_std=6.0)
    q, kb, vb = _block(3, dtype, 2, w, 4, 2, 128, gain=4.0)
    out, lse = _run(cache, batch, q, kb, vb)
    _check(cache, batch, table, lens, q, kb, vb, out, lse)


@pytest.mark.parametrize("w", [5, 20, 40, 64])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_far_logits(dtype, w):
    """Logits past 2^30, where the softmax is one-hot at the largest: its value exactly."""
    lens = [400, 64]
    cache, batch, table = random_cache(9, dtype, 2, 2, 64, lens)
    cache.k_exp.copy_(torch.where(cache.k_exp == 255, 255, 127 + 30))
    q, kb, vb = _block(3, dtype, 2, w, 2, 2, 64)
    out, lse = _run(cache, batch, q, kb, vb)
    host = HostCache(cache)
    for b in range(2):
        ref, rl, a, size = attention(host, table, lens, b, 0, 0, 0, q, kb, vb)
        f = lambda t: t[b].double().cpu().numpy()  # noqa: E731
        # only rows whose two largest logits are further apart than both may be off
        k = np.concatenate([host.rows("k", 0, 0, table[b], lens[b]), f(kb)])
        err = 2 * logit_error(dtype, size, 64) + 60
        checked = 0
        for h in range(2):
            x = f(q)[:, h] @ k[:, h].T / 8
            for i in range(w):
                top = np.sort(x[i, :lens[b] + i + 1])[-2:]
                if top[1] - top[0] > err:
                    checked += 1
                    tol = tolerance(dtype, ref[i, h], a[i, h], 0, 1, 64)
                    assert (np.abs(f(out)[i, h] - ref[i, h]) <= tol).all(), (b, h, i)
        assert checked > w // 2
        le = np.abs(lse[b].double().cpu().numpy() - rl)
        assert (le <= err + 2.0 ** -22 * np.abs(rl)).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_unreadable_pages_are_skipped_and_reported(dtype):
    lens = [700, 130]
    cache, batch, table = random_cache(8, dtype, 2, 2, 96, lens)
    bad = table.copy()
    bad[0, 3], bad[0, 4], bad[1, 0] = cache.num_pages, -5, 2 ** 31 - 1
    batch = das.Batch(batch.prefix_len, torch.as_tensor(bad, device=DEV), batch.dev_error)
    host = HostCache(cache)
    for w in (8, 50):
        batch.dev_error.zero_()
        q, kb, vb = _block(3, dtype, 2, w, 2, 2, 96)
        out = das.attn_policy_q4(cache, batch, 0, 1, 1, q, kb, vb)
        assert int(batch.dev_error) == das.DEVERR_PAGE
        for b in range(2):
            keep = np.array([bad[b, i // 64] == table[b, i // 64] for i in range(lens[b])])
            ref, _, a, size = attention(host, table, lens, b, 0, 0, 0, q, kb, vb, keep=keep)
            tol = tolerance(dtype, ref, a, size, lens[b] + w, 96)
            assert (np.abs(out[b].double().cpu().numpy() - ref) <= tol).all()


def test_bad_prefix_length_is_clamped_and_reported():
    cache, batch, table = random_cache(8, BF16, 2, 1, 64, [128, 64])
    batch = das.Batch(torch.tensor([1000, -3], dtype=torch.int32, device=DEV), batch.block_table,
                      batch.dev_error)
    q, kb, vb = _block(3, BF16, 2, 2, 1, 1, 64)
    out, lse = _run(cache, batch, q, kb, vb)
    assert int(batch.dev_error) == das.DEVERR_PREFIX
    _check(cache, batch, table, [128, 0], q, kb, vb, out, lse)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("w", [3, 40])
def test_a_visible_nan_stays_in_its_sequence_head_and_dims(dtype, w):
    lens = [100, 100]
    cache, batch, table = random_cache(8, dtype, 2, 2, 64, lens)
    x = _block(3, dtype, 2, w, 2, 2, 64)
    clean = das.attn_policy_q4(cache, batch, 0, 1, 1, *x)
    cache.v_exp[0, 0, 1, int(table[0, 1]), 2, 1, 3] = 255  # token 64 + 19, dims 32..63
    out = das.attn_policy_q4(cache, batch, 0, 1, 1, *x)
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[0, :, 1, 32:] = True
    assert torch.isnan(out[hit]).all()
    assert torch.equal(out[~hit], clean[~hit])
    cache.k_exp[0, 0, 0, int(table[1, 0]), 9, 2] = 255  # a key: all of its head's rows
    out = das.attn_policy_q4(cache, batch, 0, 1, 1, *x)
    hit[1, :, 0] = True
    assert torch.isnan(out[hit]).all()
    assert torch.equal(out[~hit], clean[~hit])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("group", [1, 2])
def test_what_later_block_positions_hold_does_not_reach_earlier_rows(dtype, group):
    """Infinities and NaN in block keys and values that a row does not see."""
    lens = [70]
    cache, batch, _ = random_cache(8, dtype, 1, 2, 64, lens)
    q, kb, vb = _block(3, dtype, 1, 40, 2 * group, 2, 64)
    clean = das.attn_policy_q4(cache, batch, 0, 1, 1, q, kb, vb)
    kb[:, 20:], vb[:, 20] = float("nan"), float("inf")
    vb[:, 35] = float("nan")
    out = das.attn_policy_q4(cache, batch, 0, 1, 1, q, kb, vb)
    assert torch.equal(out[:, :20], clean[:, :20])
    assert not torch.isfinite(out[:, 20:]).any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_an_infinite_block_value_is_infinite_where_it_is_seen(dtype):
    lens = [70]
    cache, batch, _ = random_cache(8, dtype, 1, 1, 64, lens)
    for w in (9, 40):
        q, kb, vb = _block(3, dtype, 1, w, 1, 1, 64)
        vb[0, 4, 0, 7] = -float("inf")
        out = das.attn_policy_q4(cache, batch, 0, 1, 1, q, kb, vb)
        assert (out[0, 4:, 0, 7] == -float("inf")).all()
        out[0, 4:, 0, 7] = 0
        assert torch.isfinite(out).all()


def test_repeats_streams_and_graphs_agree():
    """Equal calls give equal bits: again, on two streams at once, captured, and in two
    graphs that share a workspace and are replayed in turn."""
    lens = [2000, 333]
    cache, batch, table = random_cache(8, BF16, 2, 2, 96, lens)
    blocks = [_block(s, BF16, 2, 5, 4, 2, 96) for s in (1, 2)]
    want = [das.attn_policy_q4(cache, batch, 0, 1, 1, *x) for x in blocks]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    got = []
    for _ in range(3):
        for x, s in zip(blocks, streams):
            with torch.cuda.stream(s):
                got.append(das.attn_policy_q4(cache, batch, 0, 1, 1, *x))
    torch.cuda.synchronize()
    for i, o in enumerate(got):
        assert torch.equal(o, want[i % 2])
    ws = das.alloc_workspace_q4(cache, batch, 4, 5)
    outs, graphs = [torch.empty_like(w) for w in want], []
    for x, o in zip(blocks, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            das.attn_policy_q4(cache, batch, 0, 1, 1, *x, out=o, workspace=ws)
        graphs.append(g)
    for rep in range(4):
        for g, o, w in zip(graphs, outs, want):
            o.fill_(7)
            das.attn_policy_q4(cache, batch, 0, 1, 1, *blocks[1])  # eager work between
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, w), rep
