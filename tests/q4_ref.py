"""64-bit references of the 4-bit cache: e2m1 codes, page layouts and the commit, written
from their definitions in include/das.h, and builders of test caches."""

from __future__ import annotations

import numpy as np
import torch

from oracle import das_oracle as orc
from paper_2609_34538_amd import _lib as das

PAGE, BLOCK = 64, 32
MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
VALUES = np.concatenate([MAGNITUDES, -MAGNITUDES])
NAN_BYTE = 255


def encode(y: np.ndarray) -> np.ndarray:
    """Nearest code, ties to the even one, past 6 to 6."""
    a = np.minimum(np.abs(y), 6.0)
    hi = np.searchsorted(MAGNITUDES, a).clip(0, 7)
    lo = np.maximum(hi - 1, 0)
    d_lo, d_hi = a - MAGNITUDES[lo], MAGNITUDES[hi] - a
    code = np.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi)
    code = np.where(MAGNITUDES[hi] == a, hi, code)
    return code + 8 * np.signbit(y)


def exponents(x: np.ndarray) -> np.ndarray:
    """[..., 32] -> smallest e in -120..125 with |x| <= 7 * 2^e."""
    m = np.abs(x).max(-1)
    e = np.full(m.shape, -120)
    for step in range(-119, 126):
        e = np.where(m > 7 * 2.0 ** (step - 1), step, e)
    return e


def places(dh: int):
    """Of keys and values: [64, dh] byte of (token, dim) in a page, [64, dh / 32] byte of
    (token, block) in its exponents."""
    S = dh // 32
    k, v = np.empty((PAGE, dh), int), np.empty((PAGE, dh), int)
    ke, ve = np.empty((PAGE, S), int), np.empty((PAGE, S), int)
    for T in range(2):
        for s in range(S):
            for n in range(16):
                for e in range(2):
                    t = 32 * T + 8 * (n // 4) + 4 * e + n % 4
                    at = 4 * ((2 * T + e) * S + s)
                    ke[t, s] = n * 4 * S + at // 4
                    for g in range(4):
                        for j in range(4):
                            byte = at + j
                            k[t, 32 * s + 8 * g + 2 * j + np.arange(2)] = (
                                byte // 16 * 1024 + (16 * g + n) * 16 + byte % 16)
                for g in range(4):
                    for i in range(8):
                        t = 32 * T + 8 * g + i
                        ve[t, s] = (g * S + s) * 16 + 8 * T + i
                        v[t, 32 * s + 2 * n + np.arange(2)] = s * 1024 + (16 * g + n) * 16 + 8 * T + i
    return {"k": (k, ke), "v": (v, ve)}


class HostCache:
    """The cache's arrays on the host, with element access by (plane, layer, head)."""

    def __init__(self, cache: das.Quant4Cache):
        flat = lambda t: t.cpu().numpy().copy().reshape(*t.shape[:4], -1)  # noqa: E731
        self.dh = cache.head_dim
        self.pool = {"k": flat(cache.k_pool), "v": flat(cache.v_pool)}
        self.exp = {"k": flat(cache.k_exp), "v": flat(cache.v_exp)}
        self.at = places(self.dh)

    def rows(self, side, plane, layer, pages, n):
        """[n, Hkv, dh] elements of the first n positions on `pages`."""
        pages = np.asarray(pages, dtype=np.int64)[: -(-n // PAGE)]
        at, e_at = self.at[side]
        codes = self.pool[side][plane, layer][:, pages][..., at]        # [H, pg, 64, dh]
        codes = codes >> (4 * (np.arange(self.dh) % 2)) & 15
        e = self.exp[side][plane, layer][:, pages][..., e_at].astype(np.float64)
        scale = np.where(e == NAN_BYTE, np.nan, 2.0 ** (e - 127))
        x = VALUES[codes] * np.repeat(scale, BLOCK, axis=-1)
        return x.reshape(x.shape[0], -1, self.dh)[:, :n].transpose(1, 0, 2)

    def write(self, side, plane, layer, page, t, x):
        """Elements x [Hkv, dh] of one token, as the commit stores them."""
        at, e_at = self.at[side]
        x = x.reshape(x.shape[0], -1, BLOCK)
        fine = np.isfinite(x).all(-1)
        e = exponents(np.where(fine[..., None], x, 0.0))
        codes = encode(np.where(fine[..., None], x, 0.0) * 2.0 ** -e[..., None]).reshape(x.shape[0], -1)
        pool, exp = self.pool[side][plane, layer, :, page], self.exp[side][plane, layer, :, page]
        pool[:, at[t, 0::2]] = codes[:, 0::2] + 16 * codes[:, 1::2]
        exp[:, e_at[t]] = np.where(fine, e + 127, NAN_BYTE)

    def commit(self, table, lens, k_new, v_new, num):
        """The commit of das_kv_append_q4 on these arrays (sources in 64 bits)."""
        for side, new in (("k", k_new), ("v", v_new)):
            for p in range(new.shape[0]):
                for la in range(new.shape[1]):
                    for b, (s, n) in enumerate(zip(lens, num)):
                        for i in range(n):
                            page = table[b][(s + i) // PAGE]
                            if 0 <= page < self.pool[side].shape[3]:
                                self.write(side, p, la, page, (s + i) % PAGE, new[p, la, b, i])


def random_cache(seed, dtype, B, hkv, dh, lens, spare=0, layers=1, nk=1, nv=1, spread=0,
                 k_std=1.0, garbage=True):
    """A cache of quantised random elements (blocks' exponents over +-spread), the tables of
    sequences of `lens` on shuffled pages, and NaN exponents beside any codes in every place
    that holds no token. Returns (cache, batch, table [B, pages])."""
    rng = np.random.default_rng(seed)
    n = [max(1, -(-(s + spare) // PAGE)) for s in lens]
    total, S = sum(n) + 2, dh // 32
    perm = rng.permutation(total).astype(np.int32)
    table = np.full((B, max(n)), -1, dtype=np.int32)
    cursor = 0
    for b in range(B):
        table[b, :n[b]] = perm[cursor:cursor + n[b]]
        cursor += n[b]
    at = places(dh)
    out = {}
    for side, planes, std in (("k", nk, k_std), ("v", nv, 1.0)):
        codes = rng.integers(0, 256, size=(planes, layers, hkv, total, 32 * dh), dtype=np.uint8)
        exps = np.full((planes, layers, hkv, total, 2 * dh), NAN_BYTE if garbage else 127, dtype=np.uint8)
        for b, s in enumerate(lens):
            for pg in range(-(-s // PAGE)):
                page, live = table[b, pg], min(PAGE, s - PAGE * pg)
                shape = (planes, layers, hkv, live, S)
                x = rng.standard_normal((*shape, BLOCK)) * std
                e = exponents(x)
                c = encode(x * 2.0 ** -e[..., None]).reshape(*shape[:-1], dh).astype(np.uint8)
                codes[..., page, at[side][0][:live, 0::2]] = c[..., 0::2] + 16 * c[..., 1::2]
                e = e + rng.integers(-spread, spread + 1, size=shape)
                exps[..., page, at[side][1][:live]] = e + 127
        out[side] = (codes, exps)
    up = lambda a: torch.as_tensor(a, device="cuda")  # noqa: E731
    (kc, ke), (vc, ve) = out["k"], out["v"]
    cache = das.Quant4Cache(up(kc).view(nk, layers, hkv, total, S, 64, 16),
                            up(vc).view(nv, layers, hkv, total, S, 64, 16),
                            up(ke).view(nk, layers, hkv, total, 16, 4 * S),
                            up(ve).view(nv, layers, hkv, total, 4, S, 16), 4,
                            {i + 1: i for i in range(nk)}, {i + 1: i for i in range(nv)}, dtype)
    batch = das.Batch(up(np.asarray(lens, dtype=np.int32)), up(table),
                      torch.zeros(1, dtype=torch.int32, device="cuda"))
    return cache, batch, table


def attention(host: HostCache, table, lens, b, layer, kplane, vplane, q, kb, vb, keep=None):
    """(out, lse, |P| |V|, largest sum of |q_i k_i| / sqrt(dh)) of sequence b in 64 bits;
    `keep` masks prefix positions."""
    k = host.rows("k", kplane, layer, table[b], lens[b])
    v = host.rows("v", vplane, layer, table[b], lens[b])
    if keep is not None:
        k, v = k[keep], v[keep]
    f = lambda t: t[b].double().cpu().numpy()  # noqa: E731
    o, lse = orc.policy_attention(f(q), k, v, f(kb), f(vb))
    a, _ = orc.policy_attention(f(q), k, np.abs(v), f(kb), np.abs(f(vb)))
    dh, G = q.shape[-1], q.shape[2] // kb.shape[2]
    kk = np.abs(np.concatenate([k, f(kb)]))            # [S + w, Hkv, dh]
    size = max(float((np.abs(f(q)) @ kk[:, h].T)[:, h * G:(h + 1) * G].max()) for h in range(kb.shape[2]))
    return o, lse, a, size / np.sqrt(dh)


def logit_error(dtype, size, dh):
    """Bound of a logit's error: roundings of the sums of |q k| <= size, of a bf16 call's dh
    products or of the up to eight of an fp32 call's parts, the scale's and the exponent's."""
    return ((dh if dtype == torch.bfloat16 else 8 * dh) + 8) * 2.0 ** -24 * size


def tolerance(dtype, ref, a, size, n, dh):
    """Bound of |out - ref|: the output's half step; and, of the sum of |p v| (a), the half
    steps of a bf16 call's bf16 probabilities and fp16 records, a logit's error (in the weight
    and in the sum), the exponential's and the sums' over n positions.

    A record holds a row's results of a part scaled so that the largest lies in 2^14 .. 2^15,
    where fp16's smallest step is 2^-24: below 2^-14 the rounding is 2^-25 whatever the result,
    2^-25 / 2^14 = 2^-39 of the row's largest in that part, which is at most the row's largest
    sum of |p v|. (A result may be that much smaller: the token with all the weight can have a
    code 0.)"""
    parts = 1 if dtype == torch.bfloat16 else 8
    inner = 2 * logit_error(dtype, size, dh) + 2 * (parts * n + 16) * 2.0 ** -24
    if dtype == torch.bfloat16:
        return (2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -11 + inner) * a * 1.01
                + 2.0 ** -39 * a.max(-1, keepdims=True) + 1e-30)
    return 2.0 ** -24 * np.abs(ref) + inner * a + 1e-30
