"""Refusals of the 4-bit cache, the norm and rotation and the sampled verification: the C
ABI's status for every bad argument, before any HIP call, and the binding's checks of
tensors."""

import ctypes

import pytest
import torch

# As in the other host checks: fake device pointers and host tensors, so GPU-less hosts only.
if torch.cuda.device_count() > 0:
    pytest.skip("host-validation checks run on GPU-less hosts", allow_module_level=True)

das = pytest.importorskip("paper_2609_34538_amd._lib")
from test_serve_validation import (BAD_BATCH, BAD_CACHE, ALIGN, DEPTH, DTYPE, FAKE, NULL, SHAPE, UNSUP,  # noqa: E402
                                   WS, _batch)

LIB = das.LIB


def _cache(**kw):
    c = das.DasCacheQ4C()
    b = c.base
    b.dtype, b.num_depths, b.num_layers, b.num_kv_heads, b.head_dim, b.num_pages = 1, 4, 2, 8, 96, 50
    b.num_k_planes, b.num_v_planes = 2, 1
    for r in range(das.MAX_DEPTH + 1):
        b.k_plane[r] = b.v_plane[r] = -1
    b.k_plane[2], b.k_plane[4], b.v_plane[4] = 0, 1, 0
    b.k_pool = b.v_pool = c.k_exp = c.v_exp = FAKE
    for k, v in kw.items():
        setattr(c if k in ("k_exp", "v_exp") else b, k, v)
    return c


def _attn(c, b, layer=0, kappa=2, nu=4, hq=16, w=8, q=FAKE, kb=FAKE, vb=FAKE, out=FAKE, lse=None, ws=FAKE,
          nbytes=None):
    if nbytes is None:
        nbytes = max(LIB.das_attn_q4_workspace_bytes(ctypes.byref(c), ctypes.byref(b), hq, w), 256)
    return LIB.das_attn_q4(ctypes.byref(c), ctypes.byref(b), layer, kappa, nu, hq, w, q, kb, vb, out, lse, ws,
                           nbytes, None)


OUT = FAKE + (1 << 40)


def _append(c, b, k=FAKE, v=FAKE, w=8, num=FAKE, out=None):
    return LIB.das_kv_append_q4(ctypes.byref(c), ctypes.byref(b), k, v, w, num, out, None)


def _read(c, b, first=FAKE, num=FAKE, w=8, k=FAKE, v=OUT):
    return LIB.das_kv_read_q4(ctypes.byref(c), ctypes.byref(b), first, num, w, k, v, None)


@pytest.mark.parametrize("kw,status", BAD_CACHE + [(dict(k_exp=FAKE + 4), ALIGN)])
def test_cache_refusals(kw, status):
    c, b = _cache(**kw), _batch()
    assert _attn(c, b) == status
    assert LIB.das_attn_q4_workspace_bytes(ctypes.byref(c), ctypes.byref(b), 16, 8) == 0
    assert _append(c, b) == status and _read(c, b) == status


@pytest.mark.parametrize("kw,status", BAD_BATCH)
def test_batch_refusals(kw, status):
    c, b = _cache(), _batch(**kw)
    assert _attn(c, b) == status and _append(c, b) == status and _read(c, b) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), NULL), (dict(kb=None), NULL), (dict(vb=None), NULL), (dict(out=None), NULL),
    (dict(q=FAKE + 8), ALIGN), (dict(out=FAKE + 4), ALIGN), (dict(lse=FAKE + 2), ALIGN), (dict(layer=2), SHAPE),
    (dict(layer=-1), SHAPE), (dict(kappa=0), DEPTH), (dict(kappa=5), DEPTH), (dict(kappa=3), DEPTH),
    (dict(nu=2), DEPTH), (dict(hq=12), SHAPE), (dict(hq=0), SHAPE), (dict(hq=72), UNSUP), (dict(w=0), SHAPE),
    (dict(w=65), SHAPE), (dict(ws=None), WS), (dict(ws=FAKE + 128), WS), (dict(nbytes=0), WS)])
def test_attention_refusals(kw, status):
    assert _attn(_cache(), _batch(), **kw) == status


def test_null_structs():
    c, b = _cache(), _batch()
    a = (0, 2, 4, 16, 8, *[FAKE] * 4, None, FAKE, 1 << 20, None)
    assert LIB.das_attn_q4(None, ctypes.byref(b), *a) == NULL
    assert LIB.das_attn_q4(ctypes.byref(c), None, *a) == NULL
    assert LIB.das_kv_append_q4(None, ctypes.byref(b), FAKE, FAKE, 8, FAKE, None, None) == NULL
    assert LIB.das_kv_read_q4(ctypes.byref(c), None, FAKE, FAKE, 8, FAKE, FAKE, None) == NULL
    assert LIB.das_qk_rope(None, 1, 1, *[FAKE, 0, 0] * 3, *[FAKE] * 4, None) == NULL


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(num=None), NULL), (dict(k=FAKE + 8), ALIGN),
    (dict(v=FAKE + 4), ALIGN), (dict(w=0), SHAPE), (dict(w=65), SHAPE), (dict(out=FAKE), SHAPE),
    (dict(out=FAKE + 8), SHAPE), (dict(num=FAKE + 1), ALIGN), (dict(out=FAKE + 2), ALIGN)])
def test_append_refusals(kw, status):
    assert _append(_cache(), _batch(), **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(first=None), NULL), (dict(num=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL),
    (dict(first=FAKE + 2), ALIGN), (dict(num=FAKE + 1), ALIGN), (dict(k=FAKE + 8), ALIGN), (dict(v=OUT + 4), ALIGN),
    (dict(w=0), SHAPE), (dict(w=(1 << 20) + 1), SHAPE), (dict(v=FAKE), SHAPE),
    (dict(v=FAKE + 2 * 2 * 3 * 8 * 8 * 96 * 2 - 16), SHAPE), (dict(k=OUT + 16), SHAPE)])
def test_read_refusals(kw, status):
    assert _read(_cache(), _batch(), **kw) == status


@pytest.mark.parametrize("kw", [dict(num_layers=1 << 30), dict(num_k_planes=1 << 30), dict(num_v_planes=1 << 25),
                                dict(num_layers=2 ** 31 - 1, num_kv_heads=65535, num_k_planes=2 ** 31 - 1)])
def test_grids_that_are_too_large(kw):
    assert _append(_cache(**kw), _batch()) == SHAPE and _read(_cache(**kw), _batch()) == SHAPE
    assert _read(_cache(num_kv_heads=65535), _batch(batch=65535), w=1 << 20) == SHAPE


def test_workspace_grows_with_the_call():
    c, b = _cache(), _batch(max_pages_per_seq=400)
    n = lambda hq, w: LIB.das_attn_q4_workspace_bytes(ctypes.byref(c), ctypes.byref(b), hq, w)  # noqa: E731
    assert 0 < n(8, 1) < n(8, 16) < n(64, 16) and n(8, 1) % 256 == 0
    a = LIB.das_sampled_accept_workspace_bytes
    assert 0 < a(1, 1, 1) < a(2, 8, 100000) < a(2, 8, 1 << 20) and a(3, 7, 5000) % 256 == 0
    assert a(0, 1, 1) == a(65536, 1, 1) == a(1, 0, 1) == a(1, 65, 1) == a(1, 1, 0) == a(1, 1, (1 << 20) + 1) == 0


ROPE = dict(dtype=1, hq=4, hkv=2, dh=64, rd=64, inter=0, each=0, eps=1e-6, freq=FAKE * 3, qw=FAKE * 4, kw=FAKE * 5,
            B=3, w=5, q=FAKE * 16, qb=5 * 512, qt=512, k=FAKE * 16 + 512, kb=5 * 512, kt=512, v=FAKE * 16 + 768,
            vb=5 * 512, vt=512, pos=FAKE * 6, qo=FAKE * 32, ko=FAKE * 33, vo=FAKE * 34)


def _rope(**kw):
    a = {**ROPE, **kw}
    c = das.DasRopeC(a["dtype"], a["hq"], a["hkv"], a["dh"], a["rd"], a["inter"], a["each"], a["eps"], a["freq"],
                     a["qw"], a["kw"])
    return LIB.das_qk_rope(ctypes.byref(c), a["B"], a["w"], a["q"], a["qb"], a["qt"], a["k"], a["kb"], a["kt"], a["v"],
                           a["vb"], a["vt"], a["pos"], a["qo"], a["ko"], a["vo"], None)


DENSE = dict(q=FAKE * 16, qb=5 * 256, qt=256, k=FAKE * 17, kb=5 * 128, kt=128, v=None, vb=0, vt=0, vo=None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(qo=None), NULL), (dict(ko=None), NULL), (dict(vo=None), NULL),
    (dict(v=None), NULL), (dict(freq=None), NULL), (dict(pos=None), NULL), (dict(dtype=2), DTYPE),
    (dict(dh=80), SHAPE), (dict(rd=66), SHAPE), (dict(rd=80), SHAPE), (dict(rd=-16), SHAPE), (dict(rd=8), SHAPE),
    (dict(hq=0), SHAPE), (dict(hkv=65536), SHAPE), (dict(B=0), SHAPE), (dict(B=65536), SHAPE), (dict(w=0), SHAPE),
    (dict(w=(1 << 20) + 1), SHAPE), (dict(B=64, w=1 << 18, qb=1 << 40, kb=1 << 40, vb=1 << 40), SHAPE),
    (dict(eps=-1e-6), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(eps=float("inf")), SHAPE),
    (dict(qt=255), SHAPE), (dict(qb=4 * 512 + 255), SHAPE), (dict(kt=127), SHAPE), (dict(vb=0), SHAPE),
    (dict(qt=1 << 61), SHAPE), (dict(kb=1 << 62), SHAPE),
    (dict(q=FAKE * 16 + 8), ALIGN), (dict(qo=FAKE * 32 + 4), ALIGN), (dict(qw=FAKE * 4 + 2), ALIGN),
    (dict(freq=FAKE * 3 + 2), ALIGN), (dict(pos=FAKE * 6 + 1), ALIGN), (dict(qt=516), ALIGN), (dict(vb=5 * 512 + 4), ALIGN),
    (dict(qo=FAKE * 16), SHAPE),                                  # its own input, but with gaps
    (dict(ko=FAKE * 16 + 512), SHAPE), (dict(qo=FAKE * 33 - 16), SHAPE), (dict(vo=FAKE * 33), SHAPE),
    (dict(qo=FAKE * 3 - 512), SHAPE), (dict(ko=FAKE * 4), SHAPE), (dict(vo=FAKE * 5), SHAPE), (dict(qo=FAKE * 6), SHAPE),
    (dict(DENSE, qo=FAKE * 17), SHAPE), (dict(DENSE, ko=FAKE * 16), SHAPE), (dict(DENSE, qo=FAKE * 16 + 16), SHAPE)])
def test_rope_refusals(kw, status):
    assert _rope(**kw) == status


ACCEPT = dict(B=2, w=3, V=100, dtype=0, y=FAKE, zp=FAKE, ps=100, zq=FAKE, qs=100, T=None, Tq=None, m=None, u=FAKE,
              v=FAKE, acc=FAKE, keep=FAKE, emit=None, n=None, pr=None, ws=FAKE, bytes=1 << 20, err=None)


@pytest.mark.parametrize("kw,status", [
    (dict(y=None), NULL), (dict(zp=None), NULL), (dict(u=None), NULL), (dict(v=None), NULL), (dict(acc=None), NULL),
    (dict(keep=None), NULL), (dict(dtype=2), DTYPE), (dict(B=0), SHAPE), (dict(B=65536), SHAPE), (dict(w=0), SHAPE),
    (dict(w=65), SHAPE), (dict(V=0), SHAPE), (dict(V=(1 << 20) + 1, ps=1 << 21, qs=1 << 21), SHAPE),
    (dict(ps=99), SHAPE), (dict(qs=99), SHAPE), (dict(ps=1 << 62), SHAPE), (dict(qs=1 << 62), SHAPE),
    (dict(B=65535, w=64, V=1 << 20, ps=1 << 20, qs=1 << 20, bytes=1 << 62), SHAPE),
    (dict(zp=FAKE + 2), ALIGN), (dict(dtype=1, zq=FAKE + 1), ALIGN), (dict(y=FAKE + 2), ALIGN), (dict(T=FAKE + 2), ALIGN),
    (dict(Tq=FAKE + 1), ALIGN), (dict(m=FAKE + 1), ALIGN), (dict(u=FAKE + 2), ALIGN), (dict(v=FAKE + 2), ALIGN),
    (dict(acc=FAKE + 2), ALIGN), (dict(keep=FAKE + 1), ALIGN), (dict(emit=FAKE + 2), ALIGN), (dict(n=FAKE + 3), ALIGN),
    (dict(pr=FAKE + 2), ALIGN), (dict(err=FAKE + 2), ALIGN), (dict(ws=None), WS), (dict(ws=FAKE + 128), WS),
    (dict(bytes=255), WS)])
def test_accept_refusals(kw, status):
    assert LIB.das_sampled_accept(*{**ACCEPT, **kw}.values(), None) == status


APART = dict(ACCEPT, y=FAKE * 2, zp=FAKE * 3, zq=FAKE * 4, T=FAKE * 5, Tq=FAKE * 6, m=FAKE * 7, u=FAKE * 8, v=FAKE * 9,
             acc=FAKE * 10, keep=FAKE * 11, emit=FAKE * 12, n=FAKE * 13, pr=FAKE * 14)


@pytest.mark.parametrize("out", ["acc", "keep", "emit", "n", "pr"])
@pytest.mark.parametrize("other,at", [("y", 20), ("u", 20), ("v", 4), ("T", 4), ("Tq", 4), ("m", 4), ("zp", 5 * 400 + 396),
                                      ("zq", 5 * 400 + 396), ("acc", 4), ("keep", 4), ("emit", 20), ("n", 4), ("pr", 20)])
def test_results_of_the_verification_overlap_nothing(out, other, at):
    if out != other:
        for where in (0, at):  # the first element and the last of the other
            assert LIB.das_sampled_accept(*{**APART, out: APART[other] + where}.values(), None) == SHAPE


@pytest.mark.parametrize("held", ["k_pool", "v_pool", "k_exp", "v_exp"])
def test_read_back_does_not_overlap_the_cache(held):
    at = dict(k_pool=FAKE * 16, v_pool=FAKE * 32, k_exp=FAKE * 48, v_exp=FAKE * 64)
    planes = 2 if held[0] == "k" else 1
    last = planes * 2 * 8 * 50 * (32 * 96 if held.endswith("pool") else 2 * 96) - 16
    for where in (0, last):
        assert _read(_cache(**at), _batch(), k=at[held] + where, v=FAKE * 80) == SHAPE
        assert _read(_cache(**at), _batch(), v=at[held] + where, k=FAKE * 80) == SHAPE


def _tensors():
    cache = das.Quant4Cache.empty(2, 2, 5, 64, 2, {1: 0, 2: 1}, {2: 0}, device="cpu")
    batch = das.Batch(torch.zeros(3, dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32))
    q = torch.zeros((3, 4, 4, 64), dtype=torch.bfloat16)
    return cache, batch, q, torch.zeros((3, 4, 2, 64), dtype=torch.bfloat16)


def test_binding_checks_of_the_cache():
    c = _tensors()[0]
    assert c.head_dim == 64 and c.num_pages == 5
    bad = [dict(k_pool=c.k_pool.int()), dict(k_pool=c.k_pool[0]), dict(v_pool=c.v_pool[..., :8]),
           dict(k_exp=c.k_exp[..., :4]), dict(v_exp=c.v_exp.int()), dict(dtype=torch.float16),
           dict(k_exp=c.k_exp.transpose(2, 3)), dict(v_pool=c.v_pool.transpose(4, 5).contiguous())]
    for kw in bad:
        a = dict(k_pool=c.k_pool, v_pool=c.v_pool, k_exp=c.k_exp, v_exp=c.v_exp, num_depths=2, k_plane={1: 0},
                 v_plane={2: 0})
        with pytest.raises(ValueError):
            das.Quant4Cache(**{**a, **kw})


def test_binding_checks_of_the_attention():
    cache, batch, q, kb = _tensors()
    ws = torch.empty(1 << 16, dtype=torch.uint8)
    good = dict(q=q, k_blk=kb, v_blk=kb, out=torch.empty_like(q), lse=None, workspace=ws)
    for kw in (dict(q=q.float()), dict(q=q[0]), dict(k_blk=kb[:, :3]), dict(v_blk=kb.transpose(1, 2)),
               dict(out=q.float()), dict(out=q.transpose(1, 2)), dict(lse=torch.empty((3, 4, 3))),
               dict(lse=torch.empty((3, 4, 4), dtype=torch.bfloat16)), dict(workspace=ws.int()),
               dict(workspace=ws[::2]), dict(q=torch.zeros((2, 4, 4, 64), dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            das.attn_policy_q4(cache, batch, 0, 1, 2, **{**good, **kw})
    other = das.Batch(batch.prefix_len, batch.block_table, torch.zeros(1))
    with pytest.raises(ValueError):
        das.attn_policy_q4(cache, other, 0, 1, 2, **good)


def test_binding_checks_of_commit_and_read():
    cache, batch, _, _ = _tensors()
    k, v = torch.zeros((2, 2, 3, 4, 2, 64), dtype=torch.bfloat16), torch.zeros((1, 2, 3, 4, 2, 64), dtype=torch.bfloat16)
    n = torch.zeros(3, dtype=torch.int32)
    for a in ((k[0], v, n), (k.float(), v, n), (k, k, n), (k, v, n.long()), (k, v, n[:2]),
              (k, v, n, torch.zeros(3)), (k.transpose(0, 1), v, n)):
        with pytest.raises(ValueError):
            das.kv_append_q4(cache, batch, *a)
    for a in ((n, n, k[0], v), (n, n, k.float(), v), (n, n, k, k), (n.long(), n, k, v), (n, n[:2], k, v)):
        with pytest.raises(ValueError):
            das.kv_read_q4(cache, batch, *a)


def test_binding_checks_of_the_rotation():
    q, k = torch.zeros((2, 3, 4, 64)), torch.zeros((2, 3, 2, 64))
    pos, freq, w = torch.zeros(2, dtype=torch.int32), torch.zeros(32), torch.zeros(64)
    good = dict(q=q, k=k, positions=pos, inv_freq=freq)
    for kw in (dict(q=q.half()), dict(q=q[0]), dict(k=k.bfloat16()), dict(k=k[:1]), dict(k=k[..., :32]),
               dict(q=q.transpose(1, 2)), dict(q=torch.zeros((2, 3, 4, 128))[..., ::2]), dict(positions=pos.long()),
               dict(positions=pos[:1]), dict(positions=torch.zeros((2, 2), dtype=torch.int32)),
               dict(inv_freq=freq.double()), dict(inv_freq=freq.view(4, 8)), dict(q_weight=w.bfloat16()),
               dict(k_weight=w[:32]), dict(q_out=q.transpose(1, 2)), dict(k_out=k.bfloat16()), dict(v_out=k),
               dict(v=k[:, :2]), dict(q=torch.zeros((2, 3, 4, 80))[..., :64])):
        with pytest.raises(ValueError):
            das.qk_rope(**{**good, **kw})


def test_binding_checks_of_the_verification():
    z, u, y = torch.zeros((2, 3, 50)), torch.zeros((2, 3)), torch.zeros((2, 3), dtype=torch.int32)
    f, i = torch.zeros(2), torch.zeros(2, dtype=torch.int32)
    good = dict(proposals=y, target_logits=z, uniform=u, draw=f)
    bad = [dict(target_logits=z.half()), dict(target_logits=z[0]), dict(target_logits=z.transpose(1, 2)),
           dict(target_logits=z[:, :, ::2]), dict(target_logits=z[:1].expand(2, 3, 50)), dict(draft_logits=z.bfloat16()),
           dict(draft_logits=z[:, :2]), dict(draft_logits=z.transpose(0, 1).contiguous().transpose(0, 1)),
           dict(proposals=y.long()), dict(proposals=y[:1]), dict(uniform=u.double()), dict(draw=u), dict(draw=i),
           dict(temperature=f[:1]), dict(draft_temperature=f.double()), dict(tested=f), dict(accepted=f),
           dict(num_keep=i[:1]), dict(emitted=u), dict(num_emitted=y), dict(probs=y), dict(dev_error=f),
           dict(workspace=torch.zeros(100))]
    for kw in bad:
        with pytest.raises(ValueError):
            das.sampled_accept(**{**good, **kw})


def test_the_binding_refuses_tensors_in_host_memory():
    cache, batch, q, kb = _tensors()
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    new = torch.zeros((2, 2, 3, 4, 2, 64), dtype=torch.bfloat16)
    for call in (lambda: das.attn_policy_q4(cache, batch, 0, 1, 2, q, kb, kb),
                 lambda: das.kv_append_q4(cache, batch, new, new[:1], i32(3)),
                 lambda: das.kv_read_q4(cache, batch, i32(3), i32(3), new, new[:1].clone()),
                 lambda: das.qk_rope(q, kb, i32(3), torch.zeros(32)),
                 lambda: das.sampled_accept(i32(2, 3), torch.zeros((2, 3, 50)), torch.zeros((2, 3)), torch.zeros(2))):
        with pytest.raises(ValueError, match="on a GPU"):
            call()
