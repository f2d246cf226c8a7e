"""Verification of drawn proposals against 64-bit references of its definition: counts and
tokens exactly, over vocabularies around the kernels' parts, both types, masked and special
logits, ties, greedy rows, every refusal of a value, the distribution of what is emitted,
streams and graphs."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2609_34538_amd import _lib as das

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
I32 = dict(dtype=torch.int32, device=DEV)


def share(z, T):
    """Weights relative to the largest, and their sum, in 64 bits."""
    z = np.where(np.isnan(z), -np.inf, z.astype(np.float64))
    m = z.max()
    if not (0 < T < np.inf) or m == -np.inf:
        w = np.zeros(len(z))
        w[int(np.argmax(z))] = 1.0
        return w, 1.0
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(z == m, 1.0, np.exp((z - m) / T))
    w = np.where(np.isnan(w), 0.0, w)
    return w, w.sum()


def reference(y, zp, u, v, zq=None, T=1.0, Tq=1.0, m=None):
    """(accepted, emitted tokens, their probabilities) of one sequence."""
    w, V = zp.shape
    m = w if m is None else min(max(m, 0), w)
    v = v if 0 <= v < 1 else 0.0
    tokens, probs = [], []
    for i in range(w):
        p, Zp = share(zp[i], T)
        left = p
        if i < m:
            if zq is not None:
                q, Zq = share(zq[i], Tq)
            else:
                q, Zq = np.zeros(V), 1.0
                if 0 <= y[i] < V:
                    q[y[i]] = 1.0
            inside = 0 <= y[i] < V
            if inside and 0 <= u[i] < 1 and u[i] * (q[y[i]] / Zq) < p[y[i]] / Zp:
                tokens.append(int(y[i]))
                probs.append(p[y[i]] / Zp)
                continue
            left = p * Zq - q * Zp
            left = np.where(left > 2.0 ** -40 * (p * Zq), left, 0.0)
            if left.sum() == 0:
                left = p
        run = np.cumsum(left)
        at = int(np.searchsorted(run, v * run[-1], side="right"))
        at = min(at, int(np.nonzero(left)[0][-1]))
        tokens.append(at)
        probs.append(p[at] / Zp)
        return i, tokens, probs
    return w, tokens, probs


class Call:
    def __init__(self, zp, zq=None, y=None, T=None, Tq=None, tested=None, seed=0, u=None, v=None):
        B, w, V = zp.shape
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.zp, self.zq, self.T, self.Tq, self.tested = zp, zq, T, Tq, tested
        self.y = torch.randint(0, V, (B, w), generator=g, **I32) if y is None else y
        self.u = torch.rand((B, w), generator=g, device=DEV) if u is None else u
        self.v = torch.rand((B,), generator=g, device=DEV) if v is None else v
        self.err = torch.zeros(1, **I32)
        self.out = dict(accepted=torch.full((B,), -9, **I32), num_keep=torch.full((B,), -9, **I32),
                        emitted=torch.full((B, w), -9, **I32), num_emitted=torch.full((B,), -9, **I32),
                        probs=torch.full((B, w), -9.0, device=DEV))
        self.call = das.PreparedSampledAccept(
            self.y, zp, self.u, self.v, draft_logits=zq, temperature=T, draft_temperature=Tq,
            tested=tested, dev_error=self.err, **self.out)

    def check(self, error=0):
        self.call()
        B, w, V = self.zp.shape
        host = lambda t: None if t is None else t.float().cpu().numpy() if t.is_floating_point() else t.tolist()  # noqa: E731
        zp, zq, T, Tq = host(self.zp), host(self.zq), host(self.T), host(self.Tq)
        y, m, u, v = host(self.y), host(self.tested), host(self.u), host(self.v)
        got = {n: t.cpu().numpy() for n, t in self.out.items()}
        for b in range(B):
            a, tokens, probs = reference(y[b], zp[b], u[b].astype(np.float64), float(v[b]), None if zq is None else zq[b],
                                         1.0 if T is None else float(T[b]), 1.0 if Tq is None else float(Tq[b]),
                                         None if m is None else m[b])
            n = len(tokens)
            assert got["accepted"][b] == a and got["num_keep"][b] == n and got["num_emitted"][b] == n, b
            assert got["emitted"][b].tolist() == tokens + [-9] * (w - n), b
            # one rounding to fp32 of a value good to 2^-40
            assert (np.abs(got["probs"][b, :n] - probs) <= 2.0 ** -24 * np.array(probs) + 2.0 ** -149).all(), b
            assert (got["probs"][b, n:] == -9).all()
        assert int(self.err) == error
        return got


def _logits(seed, B, w, V, dtype, noise=0.7, gain=2.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    z = torch.randn((B, w, V), generator=g, device=DEV) * gain
    d = z + noise * torch.randn((B, w, V), generator=g, device=DEV)
    return z.to(dtype), d.to(dtype)


def _drawn(seed, d, T=1.0):
    """Proposals drawn from softmax(d / T)."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    u = torch.rand(d.shape, generator=g, device=DEV).clamp(min=1e-30)
    return (d.float() / T - torch.log(-torch.log(u))).argmax(-1).int()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,w,V", [(1, 1, 1), (3, 2, 2), (5, 3, 7), (4, 4, 511), (4, 8, 513), (6, 5, 8191),
                                   (6, 5, 8192), (6, 5, 8193), (3, 64, 1000), (2, 3, 100003), (1, 2, 1 << 20)])
@pytest.mark.parametrize("draft", [True, False])
def test_matches_the_reference(dtype, B, w, V, draft):
    z, d = _logits(V, B, w, V, dtype)
    y = _drawn(1, d) if draft else d.float().argmax(-1).int()
    Call(z, d if draft else None, y).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_temperatures_and_tested(dtype):
    B, w, V = 12, 6, 3001
    z, d = _logits(4, B, w, V, dtype, noise=0.3)
    T = torch.tensor([0.0, 0.3, 1.0, 2.5, 1e-3, 1e-40, 1e30, 1.0, 0.7, 0.0, 1.0, 1.2], device=DEV)
    Tq = torch.tensor([0.0, 0.5, 1.0, 2.5, 1.0, 0.0, 1.0, 0.2, 0.7, 1.0, 0.0, 1.2], device=DEV)
    y = torch.where((Tq > 0)[:, None], _drawn(1, d, Tq.clamp(min=0.1)[:, None, None]), d.float().argmax(-1).int())
    tested = torch.tensor([6, 0, 1, 6, 3, 6, 6, 2, 5, 6, 6, 4], **I32)
    got = Call(z, d, y, T, Tq, tested).check()
    assert got["accepted"][1] == 0 and got["accepted"].max() >= 2
    Call(z, None, z.float().argmax(-1).int(), T, None, tested).check()


@pytest.mark.parametrize("offset", [1.0e6, 1.1e6, 1.3e6, -1.0e6, -1.3e6, 2.0e9])
def test_large_logits_at_a_low_temperature(offset):
    """Logits times 32 log2(e) / T on both sides of 2^30, where weights are taken in another way;
    in steps of a sixteenth and more, with parts of a row apart by more than the range."""
    B, w, V = 3, 4, 20000
    z, d = _logits(6, B, w, V, F32, gain=0.5)
    z[:, :, 9000:], d[:, :, 9000:] = z[:, :, 9000:] - 0.3 * abs(offset), d[:, :, 9000:] - 0.3 * abs(offset)
    z[1], d[1] = z[1].flip(-1), d[1].flip(-1)
    z, d, T = z + offset, d + offset, torch.full((B,), 0.05 if abs(offset) < 1e9 else 200.0, device=DEV)
    Call(z, d, _drawn(1, d, float(T[0])), T, T).check()
    Call(z, None, z.argmax(-1).int(), T).check()


def test_rows_apart_and_off_alignment():
    """Rows of a wider table, from an odd element on."""
    for dtype in (BF16, F32):
        z, d = _logits(5, 3, 4, 9001, dtype)
        wide = [torch.full((3, 4, 9100), float("nan"), dtype=dtype, device=DEV) for _ in range(2)]
        for x, src in zip(wide, (z, d)):
            x[:, :, 7:9008] = src
        y = _drawn(2, d)
        a = Call(z, d, y)
        a.check()
        b = Call(wide[0][:, :, 7:9008], wide[1][:, :, 7:9008], y)
        b.check()
        assert all(torch.equal(a.out[n], b.out[n]) for n in a.out)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_masked_and_special_logits(dtype):
    """-inf in most places, NaN, +inf, and rows that nothing is left of."""
    B, w, V = 8, 3, 9000
    z, d = _logits(6, B, w, V, dtype)
    g = torch.Generator(device=DEV).manual_seed(8)
    inf = float("inf")
    for x in (z, d):
        x.masked_fill_(torch.rand(x.shape, generator=g, device=DEV) < 0.999, -inf)
        x[:, :, 4] = 3.0
    y = _drawn(1, d)
    z[0] = -inf                                 # target rows without a logit: token 0
    d[1] = -inf                                 # draft rows without one
    z[2, 0, 8500], z[2, 0, 8600] = inf, inf     # all weight on two tokens
    d[3, 0, 4], y[3, 0] = inf, 4
    z[4, 0, 100:200], d[4, 1, :50] = float("nan"), float("nan")
    z[5, :, 4], y[5] = -inf, 4                  # proposals that the target never makes
    z[6], d[6], y[6] = -inf, -inf, 0
    z[6, :, 8999], d[6, :, 8999] = -1e30 if dtype == BF16 else -3e38, -1.0
    Call(z, d, y).check()
    Call(z, None, y).check()


def test_equal_distributions_accept_everything():
    z, _ = _logits(7, 4, 16, 5000, BF16)
    y = _drawn(1, z)
    u = torch.full((4, 16), 1 - 2.0 ** -24, device=DEV)
    got = Call(z, z.clone(), y, u=u).check()
    assert (got["accepted"] == 16).all()


@pytest.mark.parametrize("V", [4096, 16384, 3 * 4096])
def test_ties_of_equal_logits_are_exact(V):
    """Uniform rows: the borders of the draw are at multiples of 1 / V, and numbers on them
    belong to the token above."""
    B = 64
    z = torch.full((B, 1, V), 1.5, device=DEV)
    k = torch.arange(B, device=DEV) * (V // B)
    v = (k.double() / V).float() if V != 3 * 4096 else (torch.arange(B, device=DEV) / B)
    tested = torch.zeros(B, **I32)
    got = Call(z, None, None, tested=tested, v=v).check()
    assert np.array_equal(got["emitted"][:, 0], k.cpu().numpy())
    # greedy drafts under uniform targets: u below 1 / V, on it, above
    V2 = 4096
    z = torch.zeros((3, 1, V2), device=DEV)
    u = torch.tensor([1 / V2 - 2.0 ** -24, 1 / V2, 1 / V2 + 2.0 ** -24], device=DEV).view(3, 1)
    got = Call(z, None, None, u=u).check()
    assert got["accepted"].tolist() == [1, 0, 0]


@pytest.mark.parametrize("v", [0.0, 2.0 ** -24, 1 - 2.0 ** -24])
def test_the_first_and_last_draws(v):
    """Never a token without weight: leading and trailing ones are masked."""
    for dtype in (BF16, F32):
        z, d = _logits(9, 6, 2, 20000, dtype)
        z[:, :, :9000], z[:, :, 19000:] = -float("inf"), -float("inf")
        y = _drawn(1, d)
        Call(z, d, y, v=torch.full((6,), v, device=DEV)).check()
        got = Call(z, None, y, tested=torch.zeros(6, **I32), v=torch.full((6,), v, device=DEV)).check()
        assert ((got["emitted"][:, 0] >= 9000) & (got["emitted"][:, 0] < 19000)).all()


def test_swapped_logits_leave_one_token():
    """p and q differ in two tokens that changed places: the residual is the one that p
    prefers, whatever the draw."""
    z, _ = _logits(3, 32, 1, 9000, F32)
    d = z.clone()
    d[:, 0, 100], d[:, 0, 8700] = 9.0, 2.0
    z[:, 0, 100], z[:, 0, 8700] = 2.0, 9.0
    y = torch.full((32, 1), 100, **I32)
    v = torch.linspace(0, 1 - 2.0 ** -24, 32, device=DEV)
    got = Call(z, d, y, u=torch.full((32, 1), 0.9, device=DEV), v=v).check()
    assert (got["emitted"][:, 0] == 8700).all()


def test_values_out_of_range_are_reported():
    B, w, V = 8, 3, 600
    z, d = _logits(3, B, w, V, F32, noise=0.0)
    nan = float("nan")

    def call(error, **kw):
        args = dict(zp=z, zq=d, y=_drawn(1, d), u=torch.full((B, w), 0.5, device=DEV),
                    v=torch.full((B,), 0.5, device=DEV), T=None, Tq=None, tested=None)
        Call(**{**args, **kw}).check(error)

    S, TST, P = das.DEVERR_SAMPLE, das.DEVERR_TESTED, das.DEVERR_PROPOSAL
    call(0)
    for bad in (nan, -1.0, float("inf")):
        T = torch.ones(B, device=DEV)
        T[2] = bad
        call(S, T=T)
        call(S, Tq=T)
    for bad in (nan, -0.1, 1.0, float("inf")):
        u = torch.full((B, w), 0.5, device=DEV)
        u[3, 1] = bad
        call(S, u=u)
        v = torch.full((B,), 0.5, device=DEV)
        v[1] = bad
        call(0, v=v)                                    # every proposal is accepted: no draw
        call(S, v=v, tested=torch.full((B,), 1, **I32))
    for bad in (-1, V, 2 ** 31 - 1, -(2 ** 31)):
        y = _drawn(1, d)
        y[5, 2] = bad
        call(P, y=y)
        call(P, y=y, zq=None, zp=torch.zeros_like(z), u=torch.zeros((B, w), device=DEV))
        call(0, y=y, tested=torch.full((B,), 2, **I32))  # not checked
    for bad in (-1, w + 1, 2 ** 31 - 1):
        tested = torch.full((B,), 2, **I32)
        tested[0] = bad
        call(TST, tested=tested)


def test_rows_that_nobody_asks_for_are_not_read():
    """Rows behind the tested ones hold NaN and no more than the row after them matters."""
    z, d = _logits(3, 4, 6, 9000, BF16)
    y, tested = _drawn(1, d), torch.tensor([0, 1, 2, 3], **I32)
    a = Call(z, d, y, tested=tested)
    a.check()
    for b in range(4):
        z[b, b + 1:], d[b, b:] = float("nan"), float("nan")
        y[b, b:] = -5
    c = Call(z, d, y, tested=tested)
    c.call()
    assert all(torch.equal(a.out[n], c.out[n]) for n in a.out) and int(c.err) == 0


def test_emitted_tokens_are_draws_from_the_target():
    """Frequencies over 60000 sequences with a draft that differs: Pearson's statistic of
    the first emitted token against p, of 40 tokens, within 5 deviations of its mean."""
    B, V = 60000, 40
    g = torch.Generator(device=DEV).manual_seed(11)
    zp, zq = torch.randn(V, generator=g, device=DEV), torch.randn(V, generator=g, device=DEV)
    z, d = zp.expand(B, 1, V).contiguous(), zq.expand(B, 1, V).contiguous()
    y = _drawn(5, d)
    emitted = torch.empty((B, 1), **I32)
    acc, _ = das.sampled_accept(y, z, torch.rand((B, 1), generator=g, device=DEV),
                                torch.rand(B, generator=g, device=DEV), d, emitted=emitted)
    p, q = torch.softmax(zp.double(), 0), torch.softmax(zq.double(), 0)
    counts = torch.bincount(emitted[:, 0].long(), minlength=V).double()
    chi2 = float(((counts - B * p) ** 2 / (B * p)).sum())
    assert abs(chi2 - (V - 1)) < 5 * (2 * (V - 1)) ** 0.5
    rate, want = float(acc.double().mean()), float(torch.minimum(p, q).sum())
    assert abs(rate - want) < 5 * (want * (1 - want) / B) ** 0.5


def test_repeats_streams_and_graphs_agree():
    cases = []
    for seed in (1, 2):
        z, d = _logits(seed, 5, 7, 20011, BF16)
        cases.append(Call(z, d, _drawn(seed, d), seed=seed))
    for c in cases:
        c.check()
    want = [{n: t.clone() for n, t in c.out.items()} for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                c.call()
    torch.cuda.synchronize()
    graphs = []
    for c in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.call()
        graphs.append(g)
    for rep in range(4):
        for c, w, g in zip(cases, want, graphs):
            for t in c.out.values():
                t.fill_(-9)
            cases[0].call()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(c.out[n], w[n]) for n in w), rep


def test_optional_outputs():
    z, d = _logits(3, 5, 4, 700, F32)
    c = Call(z, d, _drawn(1, d))
    c.check()
    acc, keep = das.sampled_accept(c.y, z, c.u, c.v, d)
    assert torch.equal(acc, c.out["accepted"]) and torch.equal(keep, c.out["num_keep"])
