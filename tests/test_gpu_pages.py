"""das_pages_update against a plain model of it, over runs of growing, shrinking, finished
and refused sequences."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2609_34538_amd import _lib as das

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Model:
    def __init__(self, B, most, pages, seed):
        rng = np.random.default_rng(seed)
        self.table = np.full((B, most), -1, dtype=np.int64)
        self.held = [0] * B
        self.free = [int(x) for x in rng.permutation(pages)]
        self.pages, self.most = pages, most

    def update(self, lengths, first=None, w=0):
        err, slots, need = 0, [], {}
        for b, n in enumerate(lengths):
            if 0 <= n <= 64 * self.most:
                need[b] = -(-n // 64)
            else:
                err |= das.DEVERR_PREFIX
        back = [(b, c) for b in need for c in range(need[b], self.held[b])]
        for b, c in reversed(back):
            self.free.append(int(self.table[b, c]))
            self.table[b, c] = -1
            self.held[b] = min(self.held[b], need[b])
        total, there = 0, len(self.free)
        for b in need:
            more = need[b] - self.held[b]
            total += max(more, 0)
            if more > 0 and total <= there:
                for c in range(self.held[b], need[b]):
                    self.table[b, c] = self.free.pop()
                self.held[b] = need[b]
            elif more > 0:
                err |= das.DEVERR_POOL
        for b, n in enumerate(lengths):
            for i in range(w):
                pos = first[b] + i
                ok = 0 <= pos < n and pos // 64 < self.held[b]
                slots.append(int(self.table[b, pos // 64]) * 64 + pos % 64 if ok else -1)
        return err, np.array(slots).reshape(-1, w) if w else None


class Device:
    def __init__(self, m: Model):
        i32 = dict(dtype=torch.int32, device=DEV)
        self.table = torch.as_tensor(m.table, **i32).contiguous()
        self.held = torch.tensor(m.held, **i32)
        self.free = torch.full((m.pages,), -7, **i32)
        self.free[:len(m.free)] = torch.tensor(m.free, **i32)
        self.num = torch.tensor([len(m.free)], **i32)
        self.err = torch.zeros(1, **i32)

    def update(self, lengths, first=None, w=0):
        i32 = dict(dtype=torch.int32, device=DEV)
        slots = torch.full((len(lengths), w), -99, **i32) if w else None
        self.err.zero_()
        das.pages_update(torch.tensor(lengths, **i32), self.table, self.held, self.free, self.num,
                         None if first is None else torch.tensor(first, **i32), slots, self.err)
        return int(self.err), slots

    def same_as(self, m: Model):
        assert np.array_equal(self.table.cpu().numpy(), m.table)
        assert self.held.tolist() == m.held
        assert int(self.num) == len(m.free)
        assert self.free[:len(m.free)].tolist() == m.free


@pytest.mark.parametrize("B,most,pages", [(1, 1, 1), (1, 300, 200), (5, 8, 30), (63, 16, 700), (64, 4, 100),
                                          (1024, 3, 2000), (1025, 5, 3000), (2500, 9, 9000)])
def test_runs_of_updates(B, most, pages):
    rng = np.random.default_rng(B)
    m = Model(B, most, pages, 1)
    d = Device(m)
    lens = [0] * B
    for step in range(12):
        kind = step % 4
        if kind == 0:    # a step's growth
            lens = [min(n + int(rng.integers(0, 65)), 64 * most) for n in lens]
        elif kind == 1:  # anything, short and long, some out of range
            lens = [int(x) for x in rng.integers(0, 64 * most + 1, size=B)]
            if B > 4:
                lens[3], lens[4] = -1, 64 * most + 1
        elif kind == 2:  # many finish
            lens = [int(n) if rng.random() < 0.4 and 0 <= n <= 64 * most else 0 for n in lens]
        else:            # rolled back a little
            lens = [max(n - int(rng.integers(0, 70)), 0) for n in lens]
        w = int(rng.integers(1, 65)) if step % 2 else 0
        first = [int(n - rng.integers(0, 70)) for n in lens] if w else None
        err, slots = m.update(lens, first, w)
        got_err, got_slots = d.update(lens, first, w)
        assert got_err == err, step
        d.same_as(m)
        if w:
            assert np.array_equal(got_slots.cpu().numpy(), slots), step
        lens = [min(max(n, 0), 64 * most) for n in lens]


def test_a_release_undoes_a_grant():
    m = Model(200, 40, 3000, 5)
    d = Device(m)
    lens = [int(x) for x in np.random.default_rng(1).integers(0, 900, size=200)]
    d.update(lens)
    before = [t.clone() for t in (d.table, d.held, d.free, d.num)]
    for _ in range(3):
        assert d.update([n + 64 for n in lens])[0] == 0
        d.update(lens)
        for a, b in zip((d.table, d.held, d.num), (before[0], before[1], before[3])):
            assert torch.equal(a, b)
        n = int(d.num)
        assert torch.equal(d.free[:n], before[2][:n])


@pytest.mark.parametrize("num", [-1, 31, 2 ** 31 - 1, 28])
def test_a_free_list_that_cannot_be_right_moves_nothing(num):
    """Counts out of range, and one that leaves no room for what comes back."""
    m = Model(4, 8, 30, 5)
    d = Device(m)
    d.update([200, 64, 0, 1])  # 6 pages
    before = [t.clone() for t in (d.table, d.held, d.free)]
    d.num.fill_(num)
    err, slots = d.update([0, 64, 0, 1], [0, 0, 0, 0], 2)
    assert err == das.DEVERR_POOL and int(d.num) == num
    for a, b in zip((d.table, d.held, d.free), before):
        assert torch.equal(a, b)
    t = before[0].cpu().numpy()
    assert slots.tolist() == [[-1, -1], [t[1, 0] * 64, t[1, 0] * 64 + 1], [-1, -1], [t[3, 0] * 64, -1]]


def test_held_counts_out_of_range_are_left_alone():
    m = Model(3, 4, 20, 5)
    d = Device(m)
    d.update([64, 64, 64])
    d.held[1] = 9
    before = d.table.clone()
    err, slots = d.update([128, 10, 0], [0, 0, 0], 1)
    assert err == das.DEVERR_PREFIX
    assert d.held.tolist() == [2, 9, 0]
    assert torch.equal(d.table[1], before[1]) and int(slots[1, 0]) == -1


def test_graph_replays():
    m = Model(40, 10, 300, 5)
    d = Device(m)
    d.update([100] * 40)
    i32 = dict(dtype=torch.int32, device=DEV)
    grow, back = torch.full((40,), 190, **i32), torch.full((40,), 100, **i32)
    first, slots = torch.full((40,), 100, **i32), torch.empty((40, 64), **i32)
    want = Model(40, 10, 300, 5)
    want.update([100] * 40)
    _, ref = want.update([190] * 40, [100] * 40, 64)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        das.pages_update(grow, d.table, d.held, d.free, d.num, first, slots)
        das.pages_update(back, d.table, d.held, d.free, d.num)
    for _ in range(4):
        slots.fill_(-5)
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(slots.cpu().numpy(), ref)
        assert d.held.tolist() == [2] * 40
