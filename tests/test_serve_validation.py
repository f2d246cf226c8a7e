"""Refusals of the 8-bit cache, the sampler and the page tables: the C ABI's status for
every bad argument, before any HIP call, and the binding's checks of tensors."""

import ctypes

import pytest
import torch

# As in the other host checks: fake device pointers and host tensors, so GPU-less hosts only.
if torch.cuda.device_count() > 0:
    pytest.skip("host-validation checks run on GPU-less hosts", allow_module_level=True)

das = pytest.importorskip("paper_2609_34538_amd._lib")
LIB = das.LIB
NULL, SHAPE, DEPTH, DTYPE, WS, UNSUP, ALIGN = -1, -2, -3, -4, -5, -7, -8
FAKE = 0x100000  # never dereferenced


def _cache(**kw):
    c = das.DasCacheQ8C()
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


def _batch(**kw):
    b = das.DasBatchC()
    b.batch, b.max_pages_per_seq, b.prefix_len, b.block_table, b.dev_error = 3, 7, FAKE, FAKE, None
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def _attn(c, b, layer=0, kappa=2, nu=4, hq=16, w=8, q=FAKE, kb=FAKE, vb=FAKE, out=FAKE, lse=None, ws=FAKE,
          nbytes=None):
    if nbytes is None:
        nbytes = max(LIB.das_attn_q8_workspace_bytes(ctypes.byref(c), ctypes.byref(b), hq, w), 256)
    return LIB.das_attn_q8(ctypes.byref(c), ctypes.byref(b), layer, kappa, nu, hq, w, q, kb, vb, out, lse, ws,
                           nbytes, None)


BAD_CACHE = [(dict(k_pool=None), NULL), (dict(v_pool=None), NULL), (dict(k_exp=None), NULL),
             (dict(v_exp=None), NULL), (dict(k_pool=FAKE + 8), ALIGN), (dict(v_exp=FAKE + 2), ALIGN),
             (dict(dtype=2), DTYPE), (dict(dtype=-1), DTYPE), (dict(head_dim=80), SHAPE),
             (dict(num_layers=0), SHAPE), (dict(num_kv_heads=0), SHAPE), (dict(num_kv_heads=70000), SHAPE),
             (dict(num_pages=0), SHAPE), (dict(num_depths=65), SHAPE), (dict(num_k_planes=0), SHAPE),
             (dict(num_k_planes=1), SHAPE)]
BAD_BATCH = [(dict(prefix_len=None), NULL), (dict(block_table=None), NULL), (dict(batch=0), SHAPE),
             (dict(batch=65536), SHAPE), (dict(max_pages_per_seq=0), SHAPE),
             (dict(max_pages_per_seq=(1 << 24) + 1), SHAPE), (dict(block_table=FAKE + 1), ALIGN),
             (dict(dev_error=FAKE + 2), ALIGN)]


@pytest.mark.parametrize("kw,status", BAD_CACHE)
def test_cache_refusals(kw, status):
    c, b = _cache(**kw), _batch()
    assert _attn(c, b) == status
    assert LIB.das_attn_q8_workspace_bytes(ctypes.byref(c), ctypes.byref(b), 16, 8) == 0
    assert LIB.das_kv_append_q8(ctypes.byref(c), ctypes.byref(b), FAKE, FAKE, 8, FAKE, None, None) == status


@pytest.mark.parametrize("kw,status", BAD_BATCH)
def test_batch_refusals(kw, status):
    c, b = _cache(), _batch(**kw)
    assert _attn(c, b) == status
    assert LIB.das_kv_append_q8(ctypes.byref(c), ctypes.byref(b), FAKE, FAKE, 8, FAKE, None, None) == status


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
    assert LIB.das_attn_q8(None, ctypes.byref(b), 0, 2, 4, 16, 8, *[FAKE] * 4, None, FAKE, 1 << 20, None) == NULL
    assert LIB.das_attn_q8(ctypes.byref(c), None, 0, 2, 4, 16, 8, *[FAKE] * 4, None, FAKE, 1 << 20, None) == NULL
    assert LIB.das_kv_append_q8(None, ctypes.byref(b), FAKE, FAKE, 8, FAKE, None, None) == NULL


@pytest.mark.parametrize("args,status", [
    ((None, FAKE, 8, FAKE, None), NULL), ((FAKE, None, 8, FAKE, None), NULL), ((FAKE, FAKE, 8, None, None), NULL),
    ((FAKE + 8, FAKE, 8, FAKE, None), ALIGN), ((FAKE, FAKE, 0, FAKE, None), SHAPE),
    ((FAKE, FAKE, 65, FAKE, None), SHAPE), ((FAKE, FAKE, 8, FAKE, FAKE), SHAPE),  # len_out on prefix_len
    ((FAKE, FAKE, 8, FAKE + 1, None), ALIGN), ((FAKE, FAKE, 8, FAKE, FAKE + 2), ALIGN)])
def test_append_refusals(args, status):
    assert LIB.das_kv_append_q8(ctypes.byref(_cache()), ctypes.byref(_batch()), *args, None) == status


@pytest.mark.parametrize("kw", [dict(num_layers=1 << 30), dict(num_k_planes=1 << 30), dict(num_v_planes=1 << 25),
                                dict(num_layers=2 ** 31 - 1, num_kv_heads=65535, num_k_planes=2 ** 31 - 1)])
def test_append_refuses_grids_that_are_too_large(kw):
    args = FAKE, FAKE, 8, FAKE, None, None
    assert LIB.das_kv_append_q8(ctypes.byref(_cache(**kw)), ctypes.byref(_batch()), *args) == SHAPE


def test_workspace_grows_with_the_call():
    c, b = _cache(), _batch(max_pages_per_seq=400)
    n = lambda hq, w: LIB.das_attn_q8_workspace_bytes(ctypes.byref(c), ctypes.byref(b), hq, w)  # noqa: E731
    assert 0 < n(8, 1) < n(8, 16) < n(64, 16) and n(8, 1) % 256 == 0


SAMPLE = dict(B=2, w=3, V=100, dtype=0, z=FAKE, stride=100, T=None, k=None, p=None, low=None, u=FAKE, t=FAKE,
              pr=None, err=None)


@pytest.mark.parametrize("kw,status", [
    (dict(z=None), NULL), (dict(u=None), NULL), (dict(t=None), NULL), (dict(dtype=2), DTYPE), (dict(B=0), SHAPE),
    (dict(B=65536), SHAPE), (dict(w=0), SHAPE), (dict(w=65), SHAPE), (dict(V=0), SHAPE),
    (dict(V=(1 << 20) + 1, stride=1 << 21), SHAPE), (dict(stride=99), SHAPE), (dict(stride=1 << 62), SHAPE),
    (dict(z=FAKE + 2), ALIGN), (dict(dtype=1, z=FAKE + 1), ALIGN), (dict(T=FAKE + 2), ALIGN),
    (dict(k=FAKE + 1), ALIGN), (dict(p=FAKE + 1), ALIGN), (dict(low=FAKE + 3), ALIGN), (dict(u=FAKE + 2), ALIGN),
    (dict(t=FAKE + 2), ALIGN), (dict(pr=FAKE + 2), ALIGN), (dict(err=FAKE + 2), ALIGN)])
def test_sample_refusals(kw, status):
    assert LIB.das_sample(*{**SAMPLE, **kw}.values(), None) == status


PAGES = dict(B=2, most=4, pages=9, lens=FAKE, table=FAKE, held=FAKE, free=FAKE, num=FAKE, first=FAKE, w=3,
             slots=FAKE, err=None)


@pytest.mark.parametrize("kw,status", [
    (dict(lens=None), NULL), (dict(table=None), NULL), (dict(held=None), NULL), (dict(free=None), NULL),
    (dict(num=None), NULL), (dict(first=None), NULL), (dict(slots=None), NULL), (dict(B=0), SHAPE),
    (dict(B=65536), SHAPE), (dict(most=0), SHAPE), (dict(most=1 << 25), SHAPE), (dict(B=60000, most=60000), SHAPE),
    (dict(pages=0), SHAPE), (dict(pages=1 << 25), SHAPE), (dict(w=0), SHAPE), (dict(w=65), SHAPE),
    (dict(first=None, slots=None), SHAPE), (dict(lens=FAKE + 1), ALIGN), (dict(table=FAKE + 2), ALIGN),
    (dict(slots=FAKE + 2), ALIGN), (dict(err=FAKE + 2), ALIGN)])
def test_pages_refusals(kw, status):
    assert LIB.das_pages_update(*{**PAGES, **kw}.values(), None) == status


def _tensors():
    cache = das.QuantCache.empty(2, 2, 5, 64, 2, {1: 0, 2: 1}, {2: 0}, device="cpu")
    batch = das.Batch(torch.zeros(3, dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32))
    q = torch.zeros((3, 4, 4, 64), dtype=torch.bfloat16)
    return cache, batch, q, torch.zeros((3, 4, 2, 64), dtype=torch.bfloat16)


def test_binding_checks_of_the_cache():
    c = _tensors()[0]
    bad = [dict(k_pool=c.k_pool.view(torch.uint8)), dict(k_pool=c.k_pool[0]), dict(v_pool=c.v_pool[..., :4]),
           dict(k_exp=c.k_exp[:, :, :4]), dict(v_exp=c.v_exp.int()), dict(dtype=torch.float16),
           dict(k_exp=c.k_exp.transpose(2, 3)), dict(v_pool=c.v_pool.transpose(2, 3).contiguous())]
    for kw in bad:
        a = dict(k_pool=c.k_pool, v_pool=c.v_pool, k_exp=c.k_exp, v_exp=c.v_exp, num_depths=2, k_plane={1: 0},
                 v_plane={2: 0})
        with pytest.raises(ValueError):
            das.QuantCache(**{**a, **kw})


def test_binding_checks_of_the_attention():
    cache, batch, q, kb = _tensors()
    ws = torch.empty(1 << 16, dtype=torch.uint8)
    good = dict(q=q, k_blk=kb, v_blk=kb, out=torch.empty_like(q), lse=None, workspace=ws)
    for kw in (dict(q=q.float()), dict(q=q[0]), dict(k_blk=kb[:, :3]), dict(v_blk=kb.transpose(1, 2)),
               dict(out=q.float()), dict(out=q.transpose(1, 2)), dict(lse=torch.empty((3, 4, 3))),
               dict(lse=torch.empty((3, 4, 4), dtype=torch.bfloat16)), dict(workspace=ws.int()),
               dict(workspace=ws[::2]), dict(q=torch.zeros((2, 4, 4, 64), dtype=torch.bfloat16))):
        a = {**good, **kw}
        with pytest.raises(ValueError):
            das.attn_policy_q8(cache, batch, 0, 1, 2, **a)
    other = das.Batch(batch.prefix_len, batch.block_table, torch.zeros(1))
    with pytest.raises(ValueError):
        das.attn_policy_q8(cache, other, 0, 1, 2, **good)


def test_binding_checks_of_the_commit():
    cache, batch, _, _ = _tensors()
    k, v = torch.zeros((2, 2, 3, 4, 2, 64), dtype=torch.bfloat16), torch.zeros((1, 2, 3, 4, 2, 64), dtype=torch.bfloat16)
    n = torch.zeros(3, dtype=torch.int32)
    for a in ((k[0], v, n), (k.float(), v, n), (k, k, n), (k, v, n.long()), (k, v, n[:2]),
              (k, v, n, torch.zeros(3)), (k.transpose(0, 1), v, n)):
        with pytest.raises(ValueError):
            das.kv_append_q8(cache, batch, *a)


def test_binding_checks_of_the_sampler():
    z, u = torch.zeros((2, 3, 50)), torch.zeros((2, 3))
    f, i = torch.zeros(2), torch.zeros(2, dtype=torch.int32)
    bad = [dict(logits=z.half()), dict(logits=z[0]), dict(logits=z.transpose(1, 2)), dict(logits=z[:, :, ::2]),
           dict(logits=z.transpose(0, 1)), dict(logits=z[:1].expand(2, 3, 50)), dict(uniform=u.double()),
           dict(uniform=u[:1]), dict(temperature=f[:1]), dict(temperature=f.double()), dict(top_k=f),
           dict(top_p=i), dict(min_p=u), dict(tokens=u), dict(probs=u.int()), dict(dev_error=f)]
    for kw in bad:
        with pytest.raises(ValueError):
            das.sample(**{**dict(logits=z, uniform=u), **kw})


def test_binding_checks_of_the_pages():
    i32 = dict(dtype=torch.int32)
    good = dict(lengths=torch.zeros(3, **i32), block_table=torch.zeros((3, 4), **i32),
                pages_held=torch.zeros(3, **i32), free_pages=torch.zeros(9, **i32), num_free=torch.zeros(1, **i32),
                first=torch.zeros(3, **i32), slots=torch.zeros((3, 5), **i32))
    for kw in (dict(lengths=torch.zeros(3)), dict(block_table=torch.zeros((3, 4))), dict(block_table=torch.zeros(12, **i32)),
               dict(pages_held=torch.zeros(2, **i32)), dict(num_free=torch.zeros((), **i32)), dict(first=None),
               dict(slots=None), dict(slots=torch.zeros((2, 5), **i32)), dict(slots=torch.zeros(15, **i32)),
               dict(free_pages=torch.zeros((3, 3), **i32)), dict(dev_error=torch.zeros(1))):
        with pytest.raises(ValueError):
            das.pages_update(**{**good, **kw})


def test_the_binding_refuses_tensors_in_host_memory():
    cache, batch, q, kb = _tensors()
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    new = torch.zeros((2, 2, 3, 4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="q must be"):
        das.attn_policy_q8(cache, batch, 0, 1, 2, q[0, 0], kb, kb)
    for call in (lambda: das.attn_policy_q8(cache, batch, 0, 1, 2, q, kb, kb),
                 lambda: das.kv_append_q8(cache, batch, new, new[:1], i32(3)),
                 lambda: das.sample(torch.zeros((2, 3, 50)), torch.zeros((2, 3))),
                 lambda: das.pages_update(i32(3), i32(3, 4), i32(3), i32(9), i32(1))):
        with pytest.raises(ValueError, match="on a GPU"):
            call()
