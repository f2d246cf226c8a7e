"""Prepared calls of the 8-bit cache, the sampler and the page tables go to the stream that
is current when they are called: another one than at their construction, and one that is
being captured; or to the stream that they were given."""

from __future__ import annotations

import pytest
import torch

from paper_2609_34538_amd import _lib as das

pytestmark = pytest.mark.gpu
DEV = "cuda"
B, HKV, DH, W, V, MOST = 2, 2, 64, 4, 5000, 3


class Calls:
    """Every prepared call once, on state of its own that `reset` restores."""

    def __init__(self, stream=None):
        g = torch.Generator(device=DEV).manual_seed(1)
        r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
        i32 = dict(dtype=torch.int32, device=DEV)
        bf = torch.bfloat16
        cache = das.QuantCache.empty(1, HKV, B * MOST, DH, 1, {1: 0}, {1: 0})
        batch = das.Batch(torch.full((B,), 100, **i32), torch.arange(B * MOST, **i32).view(B, MOST))
        q, kb, vb = (r(B, W, HKV, DH).to(bf) for _ in range(3))
        out, tokens, new_len = torch.empty_like(q), torch.empty((B, W), **i32), torch.empty(B, **i32)
        slots = torch.empty((B, W), **i32)
        held, free = torch.zeros(B, **i32), torch.arange(B * MOST, **i32)
        num, table = torch.tensor([B * MOST], **i32), torch.full((B, MOST), -1, **i32)
        ws = das.alloc_workspace_q8(cache, batch, HKV, W)
        self.state = [out, tokens, new_len, slots, held, free, num, table, cache.k_pool.view(torch.uint8),
                      cache.v_pool.view(torch.uint8), cache.k_exp, cache.v_exp]
        kw = dict(stream=stream)
        self.calls = [
            das.PreparedAppendQ8(cache, batch, kb[None, None], vb[None, None], torch.full((B,), 3, **i32), new_len, **kw),
            das.PreparedAttentionQ8(cache, batch, 0, 1, 1, q, kb, vb, out, ws, **kw),
            das.PreparedSample(r(B, W, V), torch.rand((B, W), generator=g, device=DEV), tokens=tokens, **kw),
            das.PreparedPages(torch.full((B,), 150, **i32), table, held, free, num,
                              torch.full((B,), 100, **i32), slots, **kw)]
        self.before = [t.clone() for t in self.state]
        torch.cuda.synchronize()

    def reset(self):
        for t, b in zip(self.state, self.before):
            t.copy_(b)

    def run(self):
        for c in self.calls:
            c()

    def results(self):
        torch.cuda.synchronize()
        return [t.clone() for t in self.state]


@pytest.fixture(scope="module")
def want():
    c = Calls()
    c.run()
    return c.results()


def _same(a, b):
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_the_stream_current_at_the_call(want):
    """Work that the side stream has queued before is waited for: the reset there comes
    behind long products, and the calls read and write what it restores."""
    c = Calls()
    side, busy = torch.cuda.Stream(), torch.ones((4096, 4096), device=DEV)
    for _ in range(3):
        c.run()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(20):
                busy @ busy
            c.reset()
            c.run()
        _same(c.results(), want)


def test_a_stream_that_is_captured(want):
    c = Calls()
    c.run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run()
    for _ in range(4):
        c.reset()
        torch.cuda.synchronize()
        g.replay()
        _same(c.results(), want)


def test_a_given_stream(want):
    side, busy = torch.cuda.Stream(), torch.ones((4096, 4096), device=DEV)
    c = Calls(side)
    for _ in range(3):
        with torch.cuda.stream(side):
            for _ in range(20):
                busy @ busy
            c.reset()
        c.run()  # current: another
        _same(c.results(), want)
