"""64-bit references of the 8-bit cache: e4m3 codes, page layouts and the commit,
written from their definitions in include/das.h, and builders of test caches."""

from __future__ import annotations

import numpy as np
import torch

from oracle import das_oracle as orc
from paper_2609_34538_amd import _lib as das

PAGE, GROUP = 64, 8
NAN_CODE = 0x7f


def e4m3_values() -> np.ndarray:
    """The value of every code: sign, 4 exponent bits (bias 7), 3 mantissa bits."""
    v = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[c] = np.nan if (e, m) == (15, 7) else (-x if c & 128 else x)
    return v


VALUES = e4m3_values()
POSITIVE = VALUES[:127]  # ascending


def encode(x: np.ndarray) -> np.ndarray:
    """Nearest code of |x| <= 448, ties to the even code; NaN code for what is not finite."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    assert (a <= 448).all()
    hi = np.searchsorted(POSITIVE, a).clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    d_lo, d_hi = a - POSITIVE[lo], POSITIVE[hi] - a
    code = np.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi)
    code = np.where(POSITIVE[hi] == a, hi, code)
    code = code | np.where(np.signbit(x), 128, 0)
    return np.where(np.isfinite(x), code, NAN_CODE).astype(np.uint8)


def exponent(x: np.ndarray) -> int:
    """Smallest e in -64..119 with |x| <= 448 * 2^e for the finite elements."""
    x = np.abs(np.asarray(x, dtype=np.float64))
    m = x[np.isfinite(x)].max(initial=0.0)
    e = -64
    while e < 119 and m > 448 * 2.0 ** e:
        e += 1
    return e


def key_bytes(dh: int) -> np.ndarray:
    """[8, dh] byte of (token, dim) in a key group."""
    t, d = np.arange(GROUP)[:, None], np.arange(dh)[None]
    return d // 32 * 256 + d % 32 // 8 * 64 + t % 4 * 16 + t // 4 * 8 + d % 8


def value_bytes(dh: int) -> np.ndarray:
    t, d = np.arange(GROUP)[:, None], np.arange(dh)[None]
    return d * 8 + t


class HostCache:
    """The cache's arrays on the host, with element access by (plane, layer, head)."""

    def __init__(self, cache: das.QuantCache):
        u8 = lambda t: t.view(torch.uint8).cpu().numpy().copy()  # noqa: E731
        self.dh = cache.head_dim
        self.pool = {"k": u8(cache.k_pool), "v": u8(cache.v_pool)}
        self.pool = {s: p.reshape(p.shape[:5] + (-1,)) for s, p in self.pool.items()}
        self.exp = {"k": u8(cache.k_exp), "v": u8(cache.v_exp)}
        self.at = {"k": key_bytes(self.dh), "v": value_bytes(self.dh)}

    def rows(self, side, plane, layer, pages, n):
        """[n, Hkv, dh] elements of the first n positions on `pages`."""
        pages = np.asarray(pages, dtype=np.int64)[: -(-n // PAGE)]
        codes = self.pool[side][plane, layer][:, pages][..., self.at[side]]  # [H, pg, 8, 8, dh]
        e = self.exp[side][plane, layer][pages].transpose(1, 0, 2).astype(np.float64) - 127
        x = VALUES[codes] * (2.0 ** e)[..., None, None]
        h = x.shape[0]
        return x.reshape(h, -1, self.dh)[:, :n].transpose(1, 0, 2)

    def commit(self, table, lens, k_new, v_new, num):
        """The commit of das_kv_append_q8 on these arrays (sources in 64 bits)."""
        for side, new in (("k", k_new), ("v", v_new)):
            pool, exp, at = self.pool[side], self.exp[side], self.at[side]
            for p in range(new.shape[0]):
                for la in range(new.shape[1]):
                    for b, (s, n) in enumerate(zip(lens, num)):
                        for g in range(s // GROUP, -(-(s + n) // GROUP) if n else 0):
                            page = table[b][g // GROUP]
                            if not 0 <= page < pool.shape[3]:
                                continue
                            lo, hi = max(s - g * 8, 0), min(s + n - g * 8, 8)
                            i = g * 8 - s
                            for h in range(new.shape[4]):
                                x = new[p, la, b, i + lo:i + hi, h]
                                e = exponent(x)
                                codes = pool[p, la, h, page, g % 8]
                                if lo:
                                    had = int(exp[p, la, page, h, g % 8]) - 127
                                    e = max(e, had)
                                    if e != had:
                                        old = codes[at[:lo]]
                                        codes[at[:lo]] = encode(VALUES[old] * 2.0 ** (had - e))
                                y = np.where(np.isfinite(x), np.clip(x * 2.0 ** -e, -448, 448), x)
                                codes[at[lo:hi]] = encode(y)
                                exp[p, la, page, h, g % 8] = e + 127


def random_cache(seed, dtype, B, hkv, dh, lens, spare=0, layers=1, nk=1, nv=1, spread=0,
                 k_std=1.0, garbage=True):
    """A cache with random elements (groups' exponents over +-spread), the tables of
    sequences of `lens` on shuffled pages, and NaN codes with the largest exponent byte in
    every place that holds no token. Returns (cache, batch, table [B, pages])."""
    rng = np.random.default_rng(seed)
    n = [max(1, -(-(s + spare) // PAGE)) for s in lens]
    total = sum(n) + 2
    perm = rng.permutation(total).astype(np.int32)
    table = np.full((B, max(n)), -1, dtype=np.int32)
    cursor = 0
    for b in range(B):
        table[b, :n[b]] = perm[cursor:cursor + n[b]]
        cursor += n[b]
    out = {}
    for side, planes, std, at in (("k", nk, k_std, key_bytes(dh)), ("v", nv, 1.0, value_bytes(dh))):
        g = torch.Generator().manual_seed(seed + (side == "v"))
        codes = np.full((planes, layers, hkv, total, 8, 8 * dh), NAN_CODE, dtype=np.uint8)
        exps = np.full((planes, layers, total, hkv, 8), 255 if garbage else 127, dtype=np.uint8)
        for b, s in enumerate(lens):
            for i in range(-(-s // GROUP)):
                page, gi, live = table[b, i // 8], i % 8, min(8, s - 8 * i)
                e = -7 + rng.integers(-spread, spread + 1, size=(planes, layers, hkv))
                exps[:, :, page, :, gi] = e + 127
                x = torch.randn((planes, layers, hkv, live, dh), generator=g) * (std * 128)
                c = x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
                where = codes[:, :, :, page, gi]
                where[..., at[:live]] = c
                codes[:, :, :, page, gi] = where
        out[side] = (codes, exps)
    dev = "cuda"
    up = lambda a: torch.as_tensor(a, device=dev)  # noqa: E731
    (kc, ke), (vc, ve) = out["k"], out["v"]
    cache = das.QuantCache(up(kc).view(torch.float8_e4m3fn),
                           up(vc).view(torch.float8_e4m3fn).view(nv, layers, hkv, total, 8, dh, 8),
                           up(ke), up(ve), 4, {i + 1: i for i in range(nk)},
                           {i + 1: i for i in range(nv)}, dtype)
    batch = das.Batch(up(np.asarray(lens, dtype=np.int32)), up(table),
                      torch.zeros(1, dtype=torch.int32, device=dev))
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


def tolerance(dtype, ref, a, size, n, dh):
    """Bound of |out - ref|: the output's half step; and, of the sum of |p v| (a), the
    half steps of a bf16 call's fp16 probabilities and fp16 records, the fp32 error of a
    logit (dh + 8 roundings of sums of |q k| <= size, in the weight and in the sum), the
    exponential's and the sums' over n positions."""
    inner = 2 * (dh + 8) * 2.0 ** -24 * size + 2 * (n + 16) * 2.0 ** -24
    if dtype == torch.bfloat16:
        return 2.0 ** -8 * np.abs(ref) + (2 * 2.0 ** -11 + inner) * a * 1.01 + 1e-30
    return 2.0 ** -24 * np.abs(ref) + inner * a + 1e-30
