"""Norm and rotation of queries and keys against 64-bit references: types, head dims and
layouts, rotated shares, both pairings, far positions, strides, in place, sizes of elements
at the ends of the types' ranges, streams and graphs."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2609_34538_amd import _lib as das

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
I32 = dict(dtype=torch.int32, device=DEV)


def _f(t):
    return t.double().cpu().numpy()


def _reference(x, weight, pos, freq, eps, interleaved):
    """64-bit result of heads x [B, w, H, dh] at positions [B, w], and the sum of the
    magnitudes that went into each element."""
    x, rd = _f(x), 2 * len(freq)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + float(np.float32(eps))) * _f(weight)
    y, size = x.copy(), np.abs(x)
    if rd:
        t = pos.astype(np.float64)[..., None, None] * freq.astype(np.float64)
        i = np.arange(0, rd, 2) if interleaved else np.arange(rd // 2)
        j = i + (1 if interleaved else rd // 2)
        c, s = np.cos(t), np.sin(t)
        y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
        both = np.abs(x[..., i]) + np.abs(x[..., j])
        size[..., i] = size[..., j] = both
    return y, size


def _check(got, want, dtype):
    """The output's half step; of the magnitudes, in fp32 half steps: the root 3 (its estimate
    is good to 2 before the last step of Newton's), two products, cosine and sine, and two for
    the sum of the turned pair."""
    ref, size = want
    tol = (2.0 ** -8 if dtype == BF16 else 2.0 ** -24) * np.abs(ref) + 8.1 * 2.0 ** -24 * size + 1e-44
    err, none = np.abs(_f(got) - ref), np.isnan(ref)
    assert np.array_equal(np.isnan(_f(got)), none)
    assert (err[~none] <= tol[~none]).all(), float((err / tol)[~none].max())


def _freq(rd):
    return (10000.0 ** (-np.arange(rd // 2) * 2.0 / max(rd, 1))).astype(np.float32)


CASES = [  # dtype, B, w, hq, hkv, dh, rotary, interleaved, norm, fused
    (BF16, 1, 1, 1, 1, 64, 64, False, True, False),
    (BF16, 2, 3, 5, 5, 96, 96, False, True, True),
    (BF16, 3, 7, 55, 55, 96, 96, True, True, True),
    (BF16, 1, 130, 32, 8, 128, 128, False, False, True),
    (BF16, 4, 5, 14, 2, 128, 64, False, True, False),
    (BF16, 2, 9, 21, 3, 96, 48, True, True, True),
    (BF16, 2, 2, 9, 3, 64, 16, False, True, True),
    (BF16, 1, 4, 33, 11, 96, 0, False, True, True),
    (F32, 2, 3, 5, 5, 96, 96, False, True, True),
    (F32, 1, 17, 17, 1, 64, 32, True, True, False),
    (F32, 3, 2, 40, 10, 128, 128, True, False, True),
    (F32, 2, 1, 3, 3, 96, 80, False, True, True),
    (F32, 1, 3000, 2, 1, 64, 64, False, True, True),
    # several tokens a workgroup, the last one not full
    (BF16, 1, 1031, 1, 1, 64, 64, False, True, False),
    (BF16, 41, 53, 5, 5, 64, 64, True, True, True),
    (BF16, 700, 3, 6, 2, 96, 96, False, True, True),
    (BF16, 19, 61, 8, 4, 128, 48, False, False, True),
    (BF16, 1100, 1, 3, 1, 96, 0, False, True, True),
    (BF16, 3, 399, 8, 4, 128, 128, True, True, True),
    (F32, 2, 1025, 4, 1, 64, 16, False, True, True),
    (F32, 5, 251, 10, 3, 128, 128, True, True, True),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{str(c[0])[6:]}-{c[1]}x{c[2]}-h{c[3]}-{c[4]}-dh{c[5]}-r{c[6]}-{'i' if c[7] else 'h'}{'n' if c[8] else ''}{'f' if c[9] else ''}")
def test_matches_the_reference(case):
    dtype, B, w, hq, hkv, dh, rd, inter, norm, fused = case
    g = torch.Generator(device=DEV).manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g, device=DEV) * 2  # noqa: E731
    if fused:  # a projection's rows, with room behind them
        x = r(B, w, hq + 2 * hkv + 1, dh).to(dtype)
        q, k, v = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:-1]
    else:
        q, k, v = r(B, w, hq, dh).to(dtype), r(B, w, hkv, dh).to(dtype), None
    freq = _freq(rd)
    rng = np.random.default_rng(1)
    first = rng.integers(0, 100000, size=B)
    weights = [(1 + 0.3 * r(dh)).to(dtype) if norm else None for _ in range(2)]
    out = das.qk_rope(q, k, torch.tensor(first, **I32), torch.tensor(freq, device=DEV) if rd else None,
                      q_weight=weights[0], k_weight=weights[1], eps=1e-5, interleaved=inter, v=v)
    pos = first[:, None] + np.arange(w)
    _check(out[0], _reference(q, weights[0], pos, freq, 1e-5, inter), dtype)
    _check(out[1], _reference(k, weights[1], pos, freq, 1e-5, inter), dtype)
    if fused:
        assert torch.equal(out[2], v)
    each = das.qk_rope(q, k, torch.tensor(pos, **I32), torch.tensor(freq, device=DEV) if rd else None,
                       q_weight=weights[0], k_weight=weights[1], eps=1e-5, interleaved=inter)
    assert torch.equal(each[0], out[0]) and torch.equal(each[1], out[1])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_far_positions(dtype):
    """Angles of any int32 position: near 2^31, negative, and rows given one by one."""
    pos = np.array([[0, 1, 2 ** 24 + 1, 2 ** 31 - 1, -1, -(2 ** 31), 1_000_003]])
    g = torch.Generator(device=DEV).manual_seed(3)
    q, k = (torch.randn((1, 7, h, 64), generator=g, device=DEV).to(dtype) for h in (3, 2))
    freq = _freq(64)
    out = das.qk_rope(q, k, torch.tensor(pos, **I32), torch.tensor(freq, device=DEV))
    _check(out[0], _reference(q, None, pos, freq, 0, False), dtype)
    _check(out[1], _reference(k, None, pos, freq, 0, False), dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [2.0 ** -140, 2.0 ** -70, 2.0 ** 70, 2.0 ** 125])
def test_sizes_of_elements(dtype, scale):
    """Squares beyond fp32's range both ways; 2^-140 is 0 in bf16, a head of which has no norm
    with eps 0."""
    g = torch.Generator(device=DEV).manual_seed(3)
    x = (torch.rand((1, 2, 3, 96), generator=g, device=DEV, dtype=torch.float64) * scale).to(dtype)
    w = torch.ones(96, dtype=dtype, device=DEV)
    freq = _freq(96)
    pos = np.array([[5, 6]])
    for eps in (0.0, 1e-6):
        out = das.qk_rope(x, x.clone(), torch.tensor([5], **I32), torch.tensor(freq, device=DEV), q_weight=w,
                          k_weight=w, eps=eps)
        _check(out[0], _reference(x, w, pos, freq, eps, False), dtype)


def test_special_rows_stay_in_their_head():
    x = torch.ones((1, 2, 4, 64), dtype=BF16, device=DEV)
    w, freq = torch.ones(64, dtype=BF16, device=DEV), torch.tensor(_freq(64), device=DEV)
    clean = das.qk_rope(x, x.clone(), torch.tensor([5], **I32), freq, q_weight=w, k_weight=w)[0]
    x[0, 0, 1, 3], x[0, 1, 2, 5], x[0, 1, 3] = float("nan"), float("inf"), 0.0
    out = das.qk_rope(x, x.clone(), torch.tensor([5], **I32), freq, q_weight=w, k_weight=w)[0]
    assert torch.isnan(out[0, 0, 1]).all()
    assert torch.isnan(out[0, 1, 2, 5]) and torch.isnan(out[0, 1, 2, 37])  # its pair
    assert (out[0, 1, 2, :5] == 0).all() and (out[0, 1, 3] == 0).all()
    for b, h in ((0, 0), (0, 2), (0, 3), (1, 0), (1, 1)):
        assert torch.equal(out[0, b, h], clean[0, b, h])


def test_one_norm_alone():
    g = torch.Generator(device=DEV).manual_seed(3)
    q, k = (torch.randn((2, 3, h, 128), generator=g, device=DEV).to(BF16) for h in (4, 2))
    w = torch.full((128,), 0.5, dtype=BF16, device=DEV)
    out = das.qk_rope(q, k, torch.zeros(2, **I32), None, k_weight=w)
    assert torch.equal(out[0], q)
    _check(out[1], _reference(k, w, np.zeros((2, 3)), np.zeros(0), 1e-6, False), BF16)


@pytest.mark.parametrize("inter", [False, True])
def test_in_place_and_untouched_neighbours(inter):
    g = torch.Generator(device=DEV).manual_seed(3)
    q, k = (torch.randn((2, 50, h, 96), generator=g, device=DEV).to(BF16) for h in (12, 4))
    freq, w = torch.tensor(_freq(64), device=DEV), torch.ones(96, dtype=BF16, device=DEV)
    kw = dict(q_weight=w, k_weight=w, interleaved=inter)
    want = das.qk_rope(q, k, torch.tensor([3, 9], **I32), freq, **kw)
    room = torch.full((2 * 50 * 12 * 96 + 128,), 3.0, dtype=BF16, device=DEV)
    inner = room[64:-64].view(q.shape)
    inner.copy_(q)
    das.qk_rope(inner, k, torch.tensor([3, 9], **I32), freq, q_out=inner, k_out=k, **kw)
    assert torch.equal(inner, want[0]) and torch.equal(k, want[1])
    assert (room[:64] == 3).all() and (room[-64:] == 3).all()


def test_streams_and_graphs_agree():
    g = torch.Generator(device=DEV).manual_seed(3)
    q, k = (torch.randn((2, 8, h, 96), generator=g, device=DEV).to(BF16) for h in (12, 4))
    pos, freq = torch.tensor([3, 9], **I32), torch.tensor(_freq(96), device=DEV)
    outs = [torch.empty_like(q), torch.empty_like(k)]
    call = das.PreparedRope(q, k, pos, freq, *outs)
    want = das.qk_rope(q, k, pos, freq)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(3):
        pos.add_(1)  # positions are read when the graph runs
        want = das.qk_rope(q, k, pos, freq)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), step
