"""The calls of the 4-bit cache, the queries' and keys' norm and rotation and the sampled
verification whose time is measured, their inputs, their plain forms and their 64-bit
results.

A case is a dict of plain values:

* op "attn": attention of a block over a cache held in 4 bits (das_attn_q4), one core
  layer, prefixes of s_min..s_max tokens on randomly placed pages, `width` block
  positions, hkv KV heads of `group` query heads each. `dtype` is the type of queries,
  block keys and values, and outputs.
* op "commit": the commit of a block's accepted inputs into `k_planes` + `v_planes` planes
  of such a cache (das_kv_append_q4), counts uniform in 0..width unless `full`, from
  positions that fall anywhere in a page, and what was written read back as the values it
  stands for (das_kv_read_q4).
* op "read": `width` positions of every sequence read back from all planes and layers.
* op "rope": norms of a block's queries and keys for each head and their rotation by
  position (das_qk_rope), from a fused projection or separate ones.
* op "accept": verification of drafted tokens against the target's probabilities
  (das_sampled_accept) from given random numbers. `draft`: the proposals were drawn from
  draft logits, or taken greedily.

Run by a program that measures `run(prepare(case, seed))`; `own` tells whether the plain
form or the library's operators run.
"""

import math

import numpy as np
import torch

own = False

PAGE, BLOCK = 64, 32                # tokens of a page, elements that share a scale
MIN_EXP, MAX_EXP = -120, 125        # exponents that the commit gives to a block
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
SIGMA, DEPTH_R = 0.2, 32
EPS, THETA = 1e-6, 10000.0
NONE = 2.0 ** -40                   # a residual below this share of p counts as none
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
DEV = "cuda"


def _attn(name, dtype, batch, hkv, group, dh, s, width, k_gain=1.0, entry="call"):
    return {"name": name, "op": "attn", "dtype": dtype, "batch": batch, "hkv": hkv, "group": group,
            "head_dim": dh, "s_min": s[0], "s_max": s[1], "width": width, "k_gain": k_gain,
            "entry": entry}


def _commit(name, dtype, batch, hkv, dh, s, width, layers, k_planes, v_planes, full=False):
    return {"name": name, "op": "commit", "dtype": dtype, "batch": batch, "hkv": hkv,
            "head_dim": dh, "s_min": s[0], "s_max": s[1], "width": width, "layers": layers,
            "k_planes": k_planes, "v_planes": v_planes, "full": full}


def _read(name, dtype, batch, hkv, dh, width, layers, k_planes, v_planes):
    return {"name": name, "op": "read", "dtype": dtype, "batch": batch, "hkv": hkv,
            "head_dim": dh, "s_min": width, "s_max": width + 64, "width": width,
            "layers": layers, "k_planes": k_planes, "v_planes": v_planes}


def _rope(name, dtype, batch, width, hq, hkv, dh, rotary, interleaved=False, norm=True,
          fused=True):
    return {"name": name, "op": "rope", "dtype": dtype, "batch": batch, "width": width, "hq": hq,
            "hkv": hkv, "head_dim": dh, "rotary": rotary, "interleaved": interleaved,
            "norm": norm, "fused": fused, "s_max": 16384}


def _accept(name, dtype, batch, width, vocab, draft=True, temps="mixed"):
    return {"name": name, "op": "accept", "dtype": dtype, "batch": batch, "width": width,
            "vocab": vocab, "draft": draft, "temps": temps}


def listed():
    return [
        # the smallest call: a four-head fp32 model, one sequence, from a decode loop
        _attn("attn_tiny_fp32", "f32", 1, 4, 1, 64, (256, 256), 4, entry="prepared"),
        # one user of a 55-head looped model, a draft of 8 positions
        _attn("attn_single", "bf16", 1, 55, 1, 96, (2048, 2048), 8, entry="prepared"),
        # ordinary decoding without a draft: one token for each of a batch of users
        _attn("attn_one_token", "bf16", 24, 8, 4, 128, (1, 8191), 1),
        # few very long prefixes under a wide grouped block, 128 query rows per KV head
        _attn("attn_long_gqa", "bf16", 4, 8, 4, 128, (32768, 32768), 32, k_gain=3.0),
        # the batched DAS-Wave step's verifier
        _attn("attn_wave", "bf16", 32, 55, 1, 96, (4096, 8192), 32),
        # one sequence's accepted tokens into all 32 depths of both pools, and back
        _commit("commit_single", "bf16", 1, 55, 96, (187, 187), 8, 4, 32, 32, full=True),
        # the batched step's commit: five key planes and the mature values
        _commit("commit_wave", "bf16", 32, 55, 96, (0, 130), 32, 4, 5, 1),
        # a sequence's whole prefix, to be moved to another cache
        _read("read_prefix", "bf16", 1, 55, 96, 2005, 4, 5, 1),
        # one user's block of 8 positions, out of a fused projection
        _rope("rope_single", "bf16", 1, 8, 55, 55, 96, 96),
        # the batched step's verifier block
        _rope("rope_wave", "bf16", 32, 32, 55, 55, 96, 96),
        # one user's block of 8 drafted tokens
        _accept("accept_single", "f32", 1, 8, 65536),
        # a serving batch's block
        _accept("accept_block", "bf16", 32, 32, 65536),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choices(["attn", "commit", "read", "rope", "accept"], [0.4, 0.15, 0.05, 0.2, 0.2])[0]
    dtype = rng.choices(["bf16", "f32"], [0.75, 0.25])[0]
    hkv = rng.choice([2, 4, 5, 8, 16, 32, 40, 55])
    dh = rng.choice([64, 96, 96, 128])
    if op == "attn":
        s_max = _log_int(rng, 1, 65536)
        s_min = s_max if rng.random() < 0.3 else rng.randint(s_max // 8, s_max)
        c = _attn("", dtype, _log_int(rng, 1, 100), hkv,
                  rng.choices([1, 2, 4, 7, 8], [5, 1, 2, 1, 1])[0], dh, (s_min, s_max),
                  _log_int(rng, 1, 64), rng.choice([1.0, 1.0, 3.0]),
                  rng.choice(["call", "prepared"]))
        # no more than the largest listed case, and fp32 no more operations than a third of its
        while c["batch"] * c["hkv"] * c["s_max"] * c["head_dim"] * max(
                1, c["width"] * c["group"] / (48 if dtype == "bf16" else 16)) > 9e8:
            k = "batch" if c["batch"] > 1 else "hkv" if c["hkv"] > 2 else "s_max"
            c[k] = max(1, c[k] // 2)
            c["s_min"] = min(c["s_min"], c["s_max"])
    elif op in ("commit", "read"):
        planes = rng.choice([(32, 32), (5, 1), (2, 1), (1, 1)])
        layers = rng.choice([1, 2, 4])
        if op == "commit":
            s_max = _log_int(rng, 1, 200)
            c = _commit("", dtype, _log_int(rng, 1, 48), hkv, dh, (rng.randint(0, s_max), s_max),
                        _log_int(rng, 1, 64), layers, *planes, full=rng.random() < 0.3)
        else:
            c = _read("", dtype, _log_int(rng, 1, 16), hkv, dh, _log_int(rng, 1, 4096), layers,
                      *planes)
        while (c["batch"] * c["k_planes"] * c["layers"] * c["hkv"] * (c["width"] + 64)
               * c["head_dim"] > 3e8):
            k = "batch" if c["batch"] > 1 else "hkv" if c["hkv"] > 2 else "width"
            c[k] = max(1, c[k] // 2)
        if op == "read":
            c["s_min"], c["s_max"] = c["width"], c["width"] + 64
    elif op == "rope":
        rotary = rng.choice([dh, dh, dh // 2, 32])
        c = _rope("", dtype, _log_int(rng, 1, 64), _log_int(rng, 1, 2048),
                  hkv * rng.choice([1, 1, 2, 4, 7]), hkv, dh, rotary, rng.random() < 0.4,
                  rng.random() < 0.7, rng.random() < 0.7)
        while c["batch"] * c["width"] * (c["hq"] + 2 * c["hkv"]) * c["head_dim"] > 2.5e7:
            k = "batch" if c["batch"] > 1 else "width"
            c[k] = max(1, c[k] // 2)
    else:
        c = _accept("", dtype, _log_int(rng, 1, 64), _log_int(rng, 1, 33),
                    _log_int(rng, 500, 200000), rng.random() < 0.75,
                    rng.choice(["mixed", "mixed", "one", "warm"]))
        while c["batch"] * c["width"] * c["vocab"] > 6e7:
            k = "batch" if c["batch"] > 1 else "width"
            c[k] = max(1, c[k] // 2)
    c.pop("name", None)
    return c


# --------------------------------------------------------------------------
# The 4-bit cache. Pages of keys and of values are 32 * dh bytes of two codes each (even
# dim low), [dh / 32][64 lanes 16 g + n][16 bytes]:
#   keys: token 32 T + 8 (n / 4) + 4 e + n % 4, dims 32 s + 8 g + 2 j, + 1 are byte
#         4 ((2 T + e) * dh / 32 + s) + j of lane 16 g + n, 16 bytes a piece
#   values: token 32 T + 8 g + i, dims 32 s + 2 n, + 1 are byte 8 T + i of piece s
# and 2 * dh bytes of exponents, one for 32 dims of a token:
#   keys [16 n][(2 T + e) * dh / 32 + s], values [4 g][s][8 T + i]
# --------------------------------------------------------------------------
def _places(dh):
    """Byte of (token, pair of dims) in a page and of (token, block) in its exponents, for
    keys and values."""
    ks = dh // 32
    t = torch.arange(PAGE, device=DEV)[:, None]
    T, r = t // 32, t % 32
    d = torch.arange(0, dh, 2, device=DEV)[None]
    s = torch.arange(ks, device=DEV)[None]
    e, n = r // 4 % 2, r // 8 * 4 + r % 4
    at = (2 * T + e) * ks + d // 32
    k = at // 4 * 1024 + (16 * (d % 32 // 8) + n) * 16 + at % 4 * 4 + d % 8 // 2
    v = d // 32 * 1024 + (16 * (r // 8) + d % 32 // 2) * 16 + 8 * T + r % 8
    ke = n * 4 * ks + (2 * T + e) * ks + s
    ve = r // 8 * 16 * ks + 16 * s + 8 * T + r % 8
    return (k, ke), (v, ve)


def _exponent(amax):
    """The smallest e with amax <= 7 * 2^e, within the range of the commit."""
    f, x = torch.frexp(amax)
    e = x.to(torch.int32) - 3 + (f > 0.875).to(torch.int32)
    return torch.where(amax > 0, e, MIN_EXP).clamp(MIN_EXP, MAX_EXP)


def _quantise(x):
    """[..., dh] values -> pairs of codes [..., dh / 2] and exponent bytes [..., dh / 32]."""
    x = x.float().unflatten(-1, (-1, BLOCK))
    fine = torch.isfinite(x).all(-1)
    e = _exponent(x.abs().amax(-1))
    y = torch.ldexp(x, -e[..., None])
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75).to(torch.uint8) + (a > 1.25).to(torch.uint8)
            + (a >= 1.75).to(torch.uint8) + (a > 2.5).to(torch.uint8)
            + (a >= 3.5).to(torch.uint8) + (a > 5).to(torch.uint8))
    code = (code + 8 * torch.signbit(y).to(torch.uint8)).flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], torch.where(fine, e + 127, 255).to(torch.uint8)


def _values(codes, exps):
    """Pairs of codes [..., dh / 2] and exponent bytes [..., dh / 32] -> fp32 [..., dh]."""
    table = torch.tensor(E2M1 + [-x for x in E2M1], device=DEV)
    pair = torch.stack([table.repeat(16), table.repeat_interleave(16)], -1)
    x = pair[codes.int()].flatten(-2).unflatten(-1, (-1, BLOCK))
    scale = torch.where(exps == 255, math.nan, torch.ldexp(torch.ones((), device=DEV),
                                                           exps.int() - 127))
    return (x * scale[..., None]).flatten(-2)


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------
def prepare(case, seed):
    return {"attn": _prepare_attn, "commit": _prepare_commit, "read": _prepare_commit,
            "rope": _prepare_rope, "accept": _prepare_accept}[case["op"]](case, seed)


def _tables(case, seed, spare):
    """Prefix lengths and randomly placed pages with room for `spare` more tokens, in a
    pool and a table for sequences of the largest length."""
    rng = np.random.default_rng(seed)
    lens = rng.integers(case["s_min"], case["s_max"] + 1, size=case["batch"])
    n = np.maximum(1, -(-(lens + spare) // PAGE))
    most = max(1, -(-(case["s_max"] + spare) // PAGE))
    total = case["batch"] * most
    perm = rng.permutation(total).astype(np.int32)
    table = np.full((case["batch"], most), -1, dtype=np.int32)
    for b, at in enumerate(np.cumsum(n) - n):
        table[b, :n[b]] = perm[at:at + n[b]]
    return rng, lens.astype(np.int32), table, total


def _generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def _pool(gen, hkv, pages, dh, std, places):
    """One plane and layer of quantised normal values: codes [1, 1, hkv, pages, 32 * dh]
    and exponents [1, 1, hkv, pages, 2 * dh]."""
    pool = torch.empty((1, 1, hkv, pages, 32 * dh), dtype=torch.uint8, device=DEV)
    exps = torch.empty((1, 1, hkv, pages, 2 * dh), dtype=torch.uint8, device=DEV)
    code_at, exp_at = (p.reshape(-1) for p in places)
    for h in range(hkv):
        x = torch.randn((pages, PAGE, dh), generator=gen, device=DEV) * std
        codes, e = _quantise(x)
        pool[0, 0, h, :, code_at] = codes.flatten(1)
        exps[0, 0, h, :, exp_at] = e.flatten(1)
    return pool, exps


def _cache(s, dtype):
    from paper_2609_34538_amd import _lib as das
    nk, L, hkv, pages = s["k_pool"].shape[:4]
    nv, dh = s["v_pool"].shape[0], s["k_pool"].shape[4] // 32
    piece, ks = (dh // 32, 64, 16), dh // 32
    return das.Quant4Cache(s["k_pool"].view(nk, L, hkv, pages, *piece),
                           s["v_pool"].view(nv, L, hkv, pages, *piece),
                           s["k_exp"].view(nk, L, hkv, pages, 16, 4 * ks),
                           s["v_exp"].view(nv, L, hkv, pages, 4, ks, 16),
                           DEPTH_R, {3: nk - 1}, {DEPTH_R: nv - 1}, dtype)


def _prepare_attn(case, seed):
    dtype, dh, hkv, B, w = (DTYPES[case["dtype"]], case["head_dim"], case["hkv"], case["batch"],
                            case["width"])
    _, lens, table, pages = _tables(case, seed, 0)
    gen = _generator(seed)
    std = math.sqrt(1 + (DEPTH_R - 1) * SIGMA ** 2)  # a random walk over recurrence depth
    k_std, v_std = (case["k_gain"], std) if case["k_gain"] != 1.0 else (1.0, std)
    kp, vp = _places(dh)
    k_pool, k_exp = _pool(gen, hkv, pages, dh, k_std, kp)
    v_pool, v_exp = _pool(gen, hkv, pages, dh, v_std, vp)

    def block(heads, std):
        return (torch.randn((B, w, heads, dh), generator=gen, device=DEV) * std).to(dtype)

    hq = hkv * case["group"]
    s = {"case": case, "lens": torch.as_tensor(lens, device=DEV),
         "table": torch.as_tensor(table, device=DEV), "k_pool": k_pool, "v_pool": v_pool,
         "k_exp": k_exp, "v_exp": v_exp, "q": block(hq, 1.0), "kb": block(hkv, k_std),
         "vb": block(hkv, v_std), "lse": torch.empty((B, hq, w), device=DEV)}
    s["out"] = torch.empty_like(s["q"])
    if own:
        from paper_2609_34538_amd import _lib as das
        s["cache"] = _cache(s, dtype)
        s["batch"] = das.Batch(s["lens"], s["table"])
        s["ws"] = das.alloc_workspace_q4(s["cache"], s["batch"], hq, w)
        if case["entry"] == "prepared":
            s["call"] = das.PreparedAttentionQ4(s["cache"], s["batch"], 0, 3, DEPTH_R, s["q"],
                                                s["kb"], s["vb"], s["out"], s["ws"], lse=s["lse"])
    return s


def _prepare_commit(case, seed):
    dtype, dh, hkv, B, w = (DTYPES[case["dtype"]], case["head_dim"], case["hkv"], case["batch"],
                            case["width"])
    read = case["op"] == "read"
    rng, lens, table, pages = _tables(case, seed, 0 if read else w)
    gen = _generator(seed)
    L, nk, nv = case["layers"], case["k_planes"], case["v_planes"]
    s = {"case": case, "lens": torch.as_tensor(lens, device=DEV),
         "table": torch.as_tensor(table, device=DEV)}
    for side, planes in (("k", nk), ("v", nv)):
        # earlier tokens: any codes, with the exponents of values around 1
        s[side + "_pool"] = torch.randint(0, 256, (planes, L, hkv, pages, 32 * dh), generator=gen,
                                          dtype=torch.uint8, device=DEV)
        s[side + "_exp"] = torch.randint(124, 129, (planes, L, hkv, pages, 2 * dh), generator=gen,
                                         dtype=torch.uint8, device=DEV)
        s[side + "_read"] = torch.zeros((planes, L, B, w, hkv, dh), dtype=dtype, device=DEV)
        if not read:  # block K/V, of a scale that differs by plane as depths do
            x = torch.randn((planes, L, B, w, hkv, dh), generator=gen, device=DEV)
            depth = torch.arange(planes, device=DEV).view(-1, 1, 1, 1, 1, 1)
            s[side + "_new"] = (x * torch.sqrt(1 + depth * SIGMA ** 2)).to(dtype)
    if read:
        first = (lens - w) // 2  # positions that start anywhere in a page
        n = np.full(B, w)
    else:
        first = lens
        n = np.full(B, w) if case["full"] else rng.integers(0, w + 1, size=B)
    s["first"] = torch.as_tensor(first.astype(np.int32), device=DEV)
    s["num"] = torch.as_tensor(n.astype(np.int32), device=DEV)
    s["len_out"] = torch.empty(B, dtype=torch.int32, device=DEV)
    if own:
        from paper_2609_34538_amd import _lib as das
        cache, batch = _cache(s, dtype), das.Batch(s["lens"], s["table"])
        if not read:
            s["append"] = das.PreparedAppendQ4(cache, batch, s["k_new"], s["v_new"], s["num"],
                                               s["len_out"])
            batch = das.Batch(s["len_out"], s["table"])
        s["back"] = das.PreparedReadQ4(cache, batch, s["first"], s["num"], s["k_read"],
                                       s["v_read"])
    return s


def _prepare_rope(case, seed):
    dtype, dh, B, w, hq, hkv = (DTYPES[case["dtype"]], case["head_dim"], case["batch"],
                                case["width"], case["hq"], case["hkv"])
    gen = _generator(seed)

    def rand(*shape):
        return torch.randn(shape, generator=gen, device=DEV)

    if case["fused"]:  # one projection's output: queries, keys and values of a token
        x = (rand(B, w, hq + 2 * hkv, dh) * 1.7).to(dtype)
        q, k, v = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:]
    else:
        q, k, v = (rand(B, w, hq, dh) * 1.7).to(dtype), (rand(B, w, hkv, dh) * 1.7).to(dtype), None
    half = torch.arange(case["rotary"] // 2, dtype=torch.float64, device=DEV)
    s = {"case": case, "q": q, "k": k, "v": v,
         "first": torch.randint(0, case["s_max"] + 1, (B,), generator=gen, dtype=torch.int32,
                                device=DEV),
         "freq": (THETA ** (-2.0 * half / case["rotary"])).float(),
         "q_weight": (1 + 0.2 * rand(dh)).to(dtype) if case["norm"] else None,
         "k_weight": (1 + 0.2 * rand(dh)).to(dtype) if case["norm"] else None}
    s["q_out"], s["k_out"] = torch.empty((B, w, hq, dh), dtype=dtype, device=DEV), torch.empty(
        (B, w, hkv, dh), dtype=dtype, device=DEV)
    s["v_out"] = None if v is None else torch.empty_like(s["k_out"])
    if own:
        from paper_2609_34538_amd import _lib as das
        s["call"] = das.PreparedRope(q, k, s["first"], s["freq"], s["q_out"], s["k_out"],
                                     q_weight=s["q_weight"], k_weight=s["k_weight"],
                                     eps=EPS if case["norm"] else 0.0,
                                     interleaved=case["interleaved"], v=v, v_out=s["v_out"])
    return s


def _prepare_accept(case, seed):
    dtype, B, w, V = DTYPES[case["dtype"]], case["batch"], case["width"], case["vocab"]
    rng, gen = np.random.default_rng(seed), _generator(seed)
    z = torch.randn((B, w, V), generator=gen, device=DEV) * 2.2
    # some tens of likely tokens, as a trained model has
    at = torch.randint(0, V, (B, w, 40), generator=gen, device=DEV)
    z.scatter_add_(2, at, 4 + 5 * torch.rand((B, w, 40), generator=gen, device=DEV))
    temps = {"mixed": [0.8, 0.6, 1.0, 1.3, 0.0], "one": [1.0], "warm": [1.0, 1.5, 2.5]}
    temp = torch.as_tensor(rng.choice(temps[case["temps"]], size=B).astype(np.float32), device=DEV)
    # a shallow draft's logits: the target's with an error
    d = z + 0.5 * torch.randn((B, w, V), generator=gen, device=DEV)
    target, draft = z.to(dtype), d.to(dtype)
    if case["draft"]:  # drawn from the draft's distribution (largest of perturbed logits)
        u = torch.rand((B, w, V), generator=gen, device=DEV).clamp(min=1e-30)
        y = torch.where((temp > 0)[:, None], (draft.float() / temp.clamp(min=1e-3)[:, None, None]
                                             - torch.log(-torch.log(u))).argmax(-1),
                        draft.float().argmax(-1))
        del u
    else:
        y = draft.float().argmax(-1)
    tested = np.where(rng.random(B) < 0.5, w, rng.integers(0, w + 1, size=B))
    s = {"case": case, "target": target, "draft": draft if case["draft"] else None, "temp": temp,
         "proposals": y.int(), "tested": torch.as_tensor(tested.astype(np.int32), device=DEV),
         "uniform": torch.rand((B, w), generator=gen, device=DEV),
         "draw": torch.rand((B,), generator=gen, device=DEV),
         "accepted": torch.empty(B, dtype=torch.int32, device=DEV),
         "num_keep": torch.empty(B, dtype=torch.int32, device=DEV),
         "emitted": torch.full((B, w), -1, dtype=torch.int32, device=DEV),
         "num_emitted": torch.empty(B, dtype=torch.int32, device=DEV),
         "probs": torch.zeros((B, w), device=DEV)}
    if own:
        from paper_2609_34538_amd import _lib as das
        s["call"] = das.PreparedSampledAccept(
            s["proposals"], target, s["uniform"], s["draw"], draft_logits=s["draft"],
            temperature=temp, draft_temperature=temp if case["draft"] else None,
            tested=s["tested"], accepted=s["accepted"], num_keep=s["num_keep"],
            emitted=s["emitted"], num_emitted=s["num_emitted"], probs=s["probs"])
    return s


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------
NAMES = {"attn": ("out", "lse"), "commit": ("k_read", "v_read", "len_out"),
         "read": ("k_read", "v_read"), "rope": ("q_out", "k_out", "v_out"),
         "accept": ("accepted", "num_keep", "emitted", "num_emitted", "probs")}


def run(s):
    op = s["case"]["op"]
    if own:
        if op == "attn" and "call" not in s:
            from paper_2609_34538_amd import _lib as das
            das.attn_policy_q4(s["cache"], s["batch"], 0, 3, DEPTH_R, s["q"], s["kb"], s["vb"],
                               out=s["out"], lse=s["lse"], workspace=s["ws"])
        elif op in ("commit", "read"):
            if op == "commit":
                s["append"]()
            s["back"]()
        else:
            s["call"]()
    else:
        {"attn": _plain_attn, "commit": _plain_commit, "read": _plain_read, "rope": _plain_rope,
         "accept": _plain_accept}[op](s)
    return {n: s[n] for n in NAMES[op]}


def _plain_attn(s):
    c = s["case"]
    dh, hkv, G, B, w = c["head_dim"], c["hkv"], c["group"], c["batch"], c["width"]
    page = s["table"].clamp(min=0).long()
    S = page.shape[1] * PAGE

    def read(pool, exps, places):  # [B, hkv, S, dh] of the prefixes
        codes = pool[0, 0][:, page][..., places[0].reshape(-1)].unflatten(-1, (PAGE, -1))
        e = exps[0, 0][:, page][..., places[1].reshape(-1)].unflatten(-1, (PAGE, -1))
        return _values(codes, e).transpose(0, 1).reshape(B, hkv, S, dh)

    kp, vp = _places(dh)
    k, v = read(s["k_pool"], s["k_exp"], kp), read(s["v_pool"], s["v_exp"], vp)
    q = s["q"].float().view(B, w, hkv, G, dh).permute(0, 2, 1, 3, 4).reshape(B, hkv, w * G, dh)
    kb, vb = (t.float().transpose(1, 2) for t in (s["kb"], s["vb"]))
    pos = torch.arange(S, device=DEV)
    hidden = (pos[None] >= s["lens"][:, None])[:, None, None, :]
    row = torch.arange(w * G, device=DEV) // G
    later = torch.arange(w, device=DEV)[None] > row[:, None]
    # values behind the last token are not part of the sum, whatever they hold
    v = torch.where(hidden.transpose(-1, -2), 0.0, v)
    scale = 1 / math.sqrt(dh)
    x = torch.cat([(torch.matmul(q, k.transpose(-1, -2)) * scale).masked_fill(hidden, -math.inf),
                   (torch.matmul(q, kb.transpose(-1, -2)) * scale).masked_fill(later, -math.inf)],
                  -1)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - m)
    total = p.sum(-1, keepdim=True)
    o = (torch.matmul(p[..., :S], v) + torch.matmul(p[..., S:], vb)) / total
    lse = (m + torch.log(total)).view(B, hkv, w, G)
    s["out"].copy_(o.view(B, hkv, w, G, dh).permute(0, 2, 1, 3, 4).reshape(B, w, hkv * G, dh))
    s["lse"].copy_(lse.permute(0, 1, 3, 2).reshape(B, hkv * G, w))


def _positions(s):
    """Page and place of the block's positions [B, w], and which of them are meant."""
    w = s["case"]["width"]
    i = torch.arange(w, device=DEV)[None]
    pos = s["first"].long()[:, None] + i
    use = i < s["num"][:, None]
    page = torch.gather(s["table"].long(), 1, torch.where(use, pos // PAGE, 0))
    return page.clamp(min=0), pos % PAGE, use


def _plain_commit(s):
    dh = s["case"]["head_dim"]
    page, at, use = _positions(s)
    page, at = page[use], at[use]  # [tokens]
    heads = torch.arange(s["case"]["hkv"], device=DEV)[None, :, None]
    for side, places in zip("kv", _places(dh)):
        codes, e = _quantise(s[side + "_new"])  # [planes, L, B, w, hkv, ...]
        where = (slice(None), slice(None), heads, page[:, None, None])
        s[side + "_pool"][(*where, places[0][at][:, None])] = codes[:, :, use]
        s[side + "_exp"][(*where, places[1][at][:, None])] = e[:, :, use]
    s["len_out"].copy_(s["lens"] + s["num"])
    _plain_read(s)


def _plain_read(s):
    dh = s["case"]["head_dim"]
    page, at, use = _positions(s)
    page, at = page[use], at[use]
    heads = torch.arange(s["case"]["hkv"], device=DEV)[None, :, None]
    for side, places in zip("kv", _places(dh)):
        where = (slice(None), slice(None), heads, page[:, None, None])
        codes = s[side + "_pool"][(*where, places[0][at][:, None])]  # [planes, L, tokens, hkv, ...]
        e = s[side + "_exp"][(*where, places[1][at][:, None])]
        s[side + "_read"][:, :, use] = _values(codes, e).to(s[side + "_read"].dtype)


def _plain_rope(s):
    c = s["case"]
    rd = c["rotary"]
    pos = s["first"][:, None] + torch.arange(c["width"], device=DEV)
    angle = pos.double()[..., None, None] * s["freq"].double()  # [B, w, 1, rd / 2]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def one(x, weight, out):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
        r = x[..., :rd].unflatten(-1, (-1, 2) if c["interleaved"] else (2, -1))
        a, b = r.unbind(-1 if c["interleaved"] else -2)
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1 if c["interleaved"] else -2)
        out.copy_(torch.cat([y.flatten(-2), x[..., rd:]], -1))

    one(s["q"], s["q_weight"], s["q_out"])
    one(s["k"], s["k_weight"], s["k_out"])
    if s["v"] is not None:
        s["v_out"].copy_(s["v"])


def _plain_weights(logits, temp):
    """exp((z - max) / T) of rows [B, w, V] and their sums; one-hot rows where T is 0 and
    where there is no logit above -inf."""
    z = logits.double()
    z = torch.where(torch.isnan(z), -math.inf, z)
    best = z.amax(-1, keepdim=True)
    T = temp.double()[:, None, None]
    first = torch.zeros_like(z).scatter_(-1, z.argmax(-1, keepdim=True), 1.0)
    weight = torch.where(z == best, 1.0, torch.exp((z - best) / torch.where(T > 0, T, 1.0)))
    weight = torch.where((T > 0) & (best > -math.inf), weight, first)
    return weight, weight.sum(-1, keepdim=True)


def _plain_accept(s):
    c = s["case"]
    B, w, V = c["batch"], c["width"], c["vocab"]
    wp, zp = _plain_weights(s["target"], s["temp"])
    y = s["proposals"].long()[..., None]
    if s["draft"] is not None:
        wq, zq = _plain_weights(s["draft"], s["temp"])
    else:
        wq, zq = torch.zeros_like(wp).scatter_(-1, y, 1.0), torch.ones_like(zp)
    pos = torch.arange(w, device=DEV)[None]
    m = s["tested"][:, None]
    u = s["uniform"].double()[..., None]
    ok = (u * (torch.gather(wq, -1, y) / zq) < torch.gather(wp, -1, y) / zp)[..., 0] & (pos < m)
    a = torch.cumprod(ok.long(), -1).sum(-1)  # the leading run of accepted ones
    at = a.clamp(max=w - 1)[:, None, None]

    def row(x):
        return torch.gather(x, 1, at.expand(B, 1, x.shape[-1]))[:, 0]

    wp_a, zp_a, wq_a, zq_a = row(wp), row(zp), row(wq), row(zq)
    left = wp_a * zq_a - wq_a * zp_a
    left = torch.where(left > NONE * (wp_a * zq_a), left, 0.0)
    # past the tested proposals, and where nothing is left, the target's own distribution
    plain = (a == s["tested"])[:, None] | (left.sum(-1, keepdim=True) == 0)
    left = torch.where(plain, wp_a, left)
    up_to = torch.cumsum(left, -1)
    token = (up_to <= s["draw"].double()[:, None] * up_to[:, -1:]).sum(-1)
    # the last token that can be drawn, where rounding took the sum past it
    last = V - 1 - (left > 0).int().flip(-1).argmax(-1)
    token = torch.minimum(token, last)
    kept = (a + 1).clamp(max=w)
    tokens = torch.where(pos < a[:, None], y[..., 0], token[:, None])
    emit = pos < kept[:, None]
    probs = (torch.gather(wp, -1, tokens[..., None]) / zp)[..., 0]
    s["accepted"].copy_(a)
    s["num_keep"].copy_(kept)
    s["num_emitted"].copy_(kept)
    s["emitted"].copy_(torch.where(emit, tokens, s["emitted"]))
    s["probs"].copy_(torch.where(emit, probs, s["probs"].double()))


# --------------------------------------------------------------------------
# Bytes and operations that a pass cannot do without
# --------------------------------------------------------------------------
def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    B, w = case["batch"], case["width"]
    if case["op"] == "attn":
        mean = (case["s_min"] + case["s_max"]) / 2
        hkv, dh, G = case["hkv"], case["head_dim"], case["group"]
        cached = B * hkv * mean * 2 * (dh / 2 + dh / BLOCK)
        block = B * w * hkv * dh * es * (2 + 2 * G) + B * w * hkv * G * 4
        return {"bytes": cached + block + B * mean / PAGE * 4,
                "flops": 4 * B * w * hkv * G * dh * (mean + (w + 1) / 2)}
    if case["op"] in ("commit", "read"):
        n = w if case["op"] == "read" or case["full"] else w / 2
        dh = case["head_dim"]
        rows = (case["k_planes"] + case["v_planes"]) * case["layers"] * B * n * case["hkv"]
        times = 2 if case["op"] == "commit" else 1
        return {"bytes": times * rows * (dh * es + dh / 2 + dh / BLOCK),
                "flops": times * rows * dh * 2}
    if case["op"] == "rope":
        heads = case["hq"] + case["hkv"] * (2 if case["fused"] else 1)
        rotated = B * w * (case["hq"] + case["hkv"]) * case["head_dim"]
        return {"bytes": 2 * B * w * heads * case["head_dim"] * es, "flops": rotated * 7}
    rows = B * w * (2 if case["draft"] else 1)
    return {"bytes": rows * case["vocab"] * es + B * w * 16, "flops": rows * case["vocab"] * 4}


# --------------------------------------------------------------------------
# The same in 64 bits, from the definitions
# --------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"attn": _exact_attn, "commit": _exact_commit, "read": _exact_commit,
            "rope": _exact_rope, "accept": _exact_accept}[case["op"]](s)


def _exact_element(byte_pairs, odd, exps):
    """64-bit elements of codes: sign, two exponent bits and one of mantissa."""
    c = (byte_pairs.int() >> torch.where(odd, 4, 0)) & 15
    ex, man = c >> 1 & 3, (c & 1).double()
    size = torch.where(ex == 0, man * 0.5, (1 + man * 0.5) * 2.0 ** (ex.double() - 1))
    size = torch.where(c >= 8, -size, size)
    return torch.where(exps == 255, math.nan, size * 2.0 ** (exps.double() - 127))


def _exact_read(pool, exps, side, dh, t):
    """Elements [..., tokens, dh] of page places t [tokens] from pages [..., tokens, 32 * dh]."""
    ks = dh // 32
    d = torch.arange(dh, device=DEV)[None]
    t = t[:, None]
    if side == "k":
        word = (t // 32 * 2 + t // 4 % 2) * ks + d // 32
        n = t % 32 // 8 * 4 + t % 4
        at = word // 4 * 1024 + (d // 8 % 4 * 16 + n) * 16 + word % 4 * 4 + d // 2 % 4
        e_at = n * 4 * ks + word
    else:
        at = d // 32 * 1024 + (t // 8 % 4 * 16 + d // 2 % 16) * 16 + t // 32 * 8 + t % 8
        e_at = t // 8 % 4 * 16 * ks + d // 32 * 16 + t // 32 * 8 + t % 8
    full = pool.shape[:-2]
    return _exact_element(torch.gather(pool, -1, at.expand(*full, -1, -1)), d % 2 == 1,
                          torch.gather(exps, -1, e_at.expand(*full, -1, -1)))


def _exact_attn(s):
    c = s["case"]
    dh, hkv, G, B, w = c["head_dim"], c["hkv"], c["group"], c["batch"], c["width"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device=DEV)
    lens, table = s["lens"].tolist(), s["table"].long()
    scale = 1 / math.sqrt(dh)
    place = torch.arange(PAGE, device=DEV)
    for b in range(B):
        n = lens[b]
        pages = table[b, :-(-n // PAGE)]
        q = s["q"][b].double().view(w, hkv, G, dh).permute(1, 2, 0, 3)  # [hkv, G, w, dh]
        for h in range(hkv):
            def rows(side, blk):
                pool, exps = (s[side + name][0, 0, h, pages][:, None].expand(-1, PAGE, -1)
                              for name in ("_pool", "_exp"))
                x = _exact_read(pool, exps, side, dh, place).reshape(-1, dh)[:n]
                return torch.cat([x, blk[b, :, h].double()])

            k, v = rows("k", s["kb"]), rows("v", s["vb"])
            x = torch.matmul(q[h].reshape(-1, dh), k.T.contiguous()).view(G, w, n + w) * scale
            j = torch.arange(n + w, device=DEV) - n
            x = torch.where(j[None, :] <= torch.arange(w, device=DEV)[:, None], x, -math.inf)
            z = torch.logsumexp(x, -1)
            o = torch.matmul(torch.exp(x - z[..., None]).view(-1, n + w), v).view(G, w, dh)
            out[b, :, h * G:(h + 1) * G] = o.transpose(0, 1)
            lse[b, h * G:(h + 1) * G] = z
    return {"out": out, "lse": lse}


def _exact_rounded(x):
    """x [..., dh] as blocks of 32 elements hold it, in 64 bits: the scale is the smallest
    power of two of which the largest magnitude is at most 7, elements are rounded to the
    nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 of it, ties to the one with an even code."""
    x = x.double().unflatten(-1, (-1, BLOCK))
    size = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(size / 7))
    # the logarithm is rounded: one step either way is put right
    e = torch.where(size > 7 * 2.0 ** e, e + 1, e)
    e = torch.where(size <= 7 * 2.0 ** (e - 1), e - 1, e).clamp(MIN_EXP, MAX_EXP)
    y = (x * 2.0 ** -e).abs()
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
    y = torch.round(y / step) * step
    return (torch.copysign(y.clamp(max=6.0), x) * 2.0 ** e).flatten(-2)


def _exact_commit(s):
    c = s["case"]
    got = {"len_out": None} if c["op"] == "commit" else {}
    first, num = s["first"].tolist(), s["num"].tolist()
    for side in "kv":
        back = torch.zeros(s[side + "_read"].shape, dtype=torch.float64, device=DEV)
        for b in range(c["batch"]):
            if not num[b]:
                continue
            if c["op"] == "commit":
                back[:, :, b, :num[b]] = _exact_rounded(s[side + "_new"][:, :, b, :num[b]])
                continue
            t = torch.arange(first[b], first[b] + num[b], device=DEV)
            pages = s["table"][b].long()[t // PAGE]
            for p in range(back.shape[0]):
                for la in range(c["layers"]):
                    x = _exact_read(s[side + "_pool"][p, la][:, pages], s[side + "_exp"][p, la][:, pages],
                                    side, c["head_dim"], t % PAGE)
                    back[p, la, b] = x.transpose(0, 1)
        got[side + "_read"] = back
    return got


def _exact_rope(s):
    c = s["case"]
    rd, B, w = c["rotary"], c["batch"], c["width"]
    t = (s["first"].long()[:, None] + torch.arange(w, device=DEV)).double()
    turn = torch.polar(torch.ones((B, w, 1, rd // 2), dtype=torch.float64, device=DEV),
                       t[..., None, None] * s["freq"].double())
    if c["interleaved"]:
        i = torch.arange(0, rd, 2, device=DEV)
        j = i + 1
    else:
        i = torch.arange(rd // 2, device=DEV)
        j = i + rd // 2

    def one(x, weight):
        x = x.double()
        if weight is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS) * weight.double()
        y = x.clone()
        z = torch.complex(x[..., i], x[..., j]) * turn
        y[..., i], y[..., j] = z.real, z.imag
        return y

    return {"q_out": one(s["q"], s["q_weight"]), "k_out": one(s["k"], s["k_weight"]),
            "v_out": None if s["v"] is None else s["v"].double()}


def _exact_accept(s):
    c = s["case"]
    B, w = c["batch"], c["width"]
    if B * w * c["vocab"] > 1 << 27:
        return None
    probs = torch.zeros((B, w), dtype=torch.float64)
    temp, tested = s["temp"].tolist(), s["tested"].tolist()
    uniform, draws = s["uniform"].tolist(), s["draw"].tolist()

    def share(logits, T):
        z = logits.double().cpu().numpy()
        if T <= 0:
            p = np.zeros(len(z))
            p[int(np.argmax(z))] = 1.0
            return p
        p = np.exp((z - z.max()) / T)
        return p / p.sum()

    for b in range(B):
        for i in range(w):
            p = share(s["target"][b, i], temp[b])
            y = int(s["proposals"][b, i])
            if i < tested[b]:
                if s["draft"] is not None:
                    q = share(s["draft"][b, i], temp[b])
                else:
                    q = np.zeros(len(p))
                    q[y] = 1.0
                if uniform[b][i] * q[y] < p[y]:
                    probs[b, i] = p[y]
                    continue
                left = p - q
                left = np.where(left > NONE * p, left, 0.0)
                left = left if left.sum() > 0 else p
            else:
                left = p
            up_to = np.cumsum(left)
            at = int(np.searchsorted(up_to, draws[b] * up_to[-1], side="right"))
            probs[b, i] = p[min(at, int(np.nonzero(left)[0][-1]))]
            break
    return {"accepted": None, "num_keep": None, "emitted": None, "num_emitted": None,
            "probs": probs}
