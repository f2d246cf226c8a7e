"""A prepared call keeps the tensors that it will read and write, also where its cache and
batch objects are given others afterwards."""

import weakref

import pytest
import torch

# As in the other host checks: host tensors, so GPU-less hosts only.
if torch.cuda.device_count() > 0:
    pytest.skip("host checks run on GPU-less hosts", allow_module_level=True)

das = pytest.importorskip("paper_2609_34538_amd._lib")


def _case():
    i32 = dict(dtype=torch.int32)
    cache = das.QuantCache.empty(1, 2, 5, 64, 1, {1: 0}, {1: 0}, device="cpu")
    batch = das.Batch(torch.zeros(3, **i32), torch.zeros((3, 2), **i32), torch.zeros(1, **i32))
    q, kb = torch.zeros((3, 4, 4, 64), dtype=torch.bfloat16), torch.zeros((3, 4, 2, 64), dtype=torch.bfloat16)
    return cache, batch, q, kb


def _attention(cache, batch, q, kb):
    return das.PreparedAttentionQ8(cache, batch, 0, 1, 1, q, kb, kb, torch.empty_like(q),
                                   torch.empty(1 << 16, dtype=torch.uint8))


def _append(cache, batch, q, kb):
    return das.PreparedAppendQ8(cache, batch, kb[None, None], kb[None, None], torch.zeros(3, dtype=torch.int32))


@pytest.mark.parametrize("make", [_attention, _append])
def test_tensors_of_the_cache_and_batch_are_kept(make):
    cache, batch, q, kb = _case()
    call = make(cache, batch, q, kb)
    names = ["k_pool", "v_pool", "k_exp", "v_exp"]
    old = [weakref.ref(getattr(cache, n)) for n in names]
    old += [weakref.ref(getattr(batch, n)) for n in ("prefix_len", "block_table", "dev_error")]
    at = [r().data_ptr() for r in old]
    for n in names:
        setattr(cache, n, getattr(cache, n).clone())
    cache.refresh()
    batch.prefix_len, batch.block_table, batch.dev_error = (
        batch.prefix_len.clone(), batch.block_table.clone(), batch.dev_error.clone())
    batch.refresh()
    assert [r() is not None and r().data_ptr() for r in old] == at
    # and the call still names them
    assert call._args[0]._obj.base.k_pool == at[0] and call._args[0]._obj.v_exp == at[3]
    assert call._args[1]._obj.prefix_len == at[4] and call._args[1]._obj.dev_error == at[6]
