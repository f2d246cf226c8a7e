"""The operators together, as a decode loop uses them: pages for the block, draft and
verifier attention over the 8-bit cache, sampled predictions, acceptance, the commit in 8
bits and the release of unused pages, without a host round trip; run eagerly and as one
captured graph, and checked step by step against 64-bit references."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import das_oracle as orc
from paper_2609_34538_amd import _lib as das
from q8_ref import HostCache, attention, tolerance
from test_gpu_pages import Model
from test_gpu_sample import reference

pytestmark = pytest.mark.gpu
DEV = "cuda"
B, HKV, G, DH, L, W, V, R, MOST, PAGES = 3, 2, 2, 64, 2, 6, 401, 2, 6, 16


class Loop:
    """A model whose layers are random projections: the step's calls are what counts."""

    def __init__(self, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
        i32 = dict(dtype=torch.int32, device=DEV)
        self.cache = das.QuantCache.empty(L, HKV, PAGES, DH, R, {1: 0, R: 1}, {R: 0})
        self.table = torch.full((B, MOST), -1, **i32)
        self.held, self.lens = torch.zeros(B, **i32), torch.zeros(B, **i32)
        self.free = torch.arange(PAGES, **i32)
        self.num_free = torch.tensor([PAGES], **i32)
        self.err = torch.zeros(1, **i32)
        self.batch = das.Batch(self.lens, self.table, self.err)
        self.want, self.new_len = torch.empty(B, **i32), torch.empty(B, **i32)
        self.slots = torch.empty((B, W), **i32)
        bf = torch.bfloat16
        self.q = r(2, L, B, W, HKV * G, DH).to(bf)
        self.k_new, self.v_new = r(2, L, B, W, HKV, DH).to(bf), r(1, L, B, W, HKV, DH).to(bf)
        self.read = (r(HKV * G * DH, V) * 0.3).to(bf)
        self.y = torch.randint(0, V, (B, W), generator=g, device=DEV, dtype=torch.int32)
        self.u = torch.rand((B, W), generator=g, device=DEV)
        self.T = torch.tensor([0.8, 0.0, 1.1], device=DEV)
        self.k = torch.tensor([0, 0, 40], **i32)
        self.p = torch.tensor([0.9, 1.0, 0.95], device=DEV)
        self.out = torch.empty_like(self.q)
        self.logits = torch.empty((B, W, V), device=DEV, dtype=bf)
        self.tokens, self.acc, self.keep = torch.empty((B, W), **i32), torch.empty(B, **i32), torch.empty(B, **i32)
        self.ws = das.alloc_workspace_q8(self.cache, self.batch, HKV * G, W)

    def step(self):
        torch.add(self.lens, W, out=self.want)
        das.pages_update(self.want, self.table, self.held, self.free, self.num_free, self.lens,
                         self.slots, self.err)
        for la in range(L):
            for i, d in enumerate((1, R)):  # the draft's read, then the verifier's
                das.attn_policy_q8(self.cache, self.batch, la, d, R, self.q[i, la], self.k_new[i, la],
                                   self.v_new[0, la], out=self.out[i, la], workspace=self.ws)
        torch.matmul(self.out[1, L - 1].view(B * W, -1), self.read, out=self.logits.view(B * W, V))
        das.sample(self.logits, self.u, self.T, self.k, self.p, tokens=self.tokens, dev_error=self.err)
        das.greedy_accept(self.y, self.tokens, accepted=self.acc, num_keep=self.keep)
        das.kv_append_q8(self.cache, self.batch, self.k_new, self.v_new, self.keep, self.new_len)
        self.lens.copy_(self.new_len)
        das.pages_update(self.lens, self.table, self.held, self.free, self.num_free, dev_error=self.err)


def test_steps_against_references():
    s = Loop(1)
    pages = Model(B, MOST, PAGES, 0)
    pages.free = list(range(PAGES))
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    for n in range(9):
        lens, host = s.lens.tolist(), HostCache(s.cache)
        s.y.copy_(torch.where(torch.rand((B, W), device=DEV) < 0.7, s.tokens.clamp(0, V - 1), s.y))
        y = s.y.cpu().numpy()
        s.step()
        err, slots = pages.update([x + W for x in lens], lens, W)
        assert err == 0 and np.array_equal(s.slots.cpu().numpy(), slots)
        table = pages.table.copy()
        for la in range(L):
            for i in range(2):
                for b in range(B):
                    args = (s.q[i, la], s.k_new[i, la], s.v_new[0, la])
                    ref, _, a, size = attention(host, table, lens, b, la, i, 0, *args)
                    tol = tolerance(torch.bfloat16, ref, a, size, lens[b] + W, DH)
                    assert (np.abs(f(s.out[i, la][b]) - ref) <= tol).all(), (n, la, i, b)
        z, u = s.logits.float().cpu().numpy(), f(s.u)
        keep = []
        for b in range(B):
            tok = [reference(z[b, i], u[b, i], float(s.T[b]), int(s.k[b]), float(s.p[b]))[0] for i in range(W)]
            assert s.tokens[b].tolist() == tok
            a, _ = orc.greedy_accept(y[b].tolist(), tok, W)
            keep.append(orc.commit_count(a, W))
        assert s.keep.tolist() == keep
        host.commit(table, lens, f(s.k_new), f(s.v_new), keep)
        got = HostCache(s.cache)
        for side in "kv":
            assert np.array_equal(got.pool[side], host.pool[side]) and np.array_equal(got.exp[side], host.exp[side])
        lens = [x + k for x, k in zip(lens, keep)]
        assert s.lens.tolist() == lens
        assert pages.update(lens)[0] == 0
        assert np.array_equal(s.table.cpu().numpy(), pages.table) and s.held.tolist() == pages.held
        assert int(s.err) == 0


def test_the_captured_step_matches_eager_steps():
    a, b = Loop(2), Loop(2)
    for s in (a, b):
        s.step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.step()
    for _ in range(6):
        a.step()
        g.replay()
        torch.cuda.synchronize()
        for x, y in ((a.out, b.out), (a.tokens, b.tokens), (a.lens, b.lens), (a.table, b.table),
                     (a.cache.k_pool.view(torch.uint8), b.cache.k_pool.view(torch.uint8)),
                     (a.cache.v_exp, b.cache.v_exp), (a.num_free, b.num_free)):
            assert torch.equal(x, y)
