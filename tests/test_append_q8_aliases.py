"""das_kv_append_q8 refuses a len_out that shares elements with the lengths or the counts,
which other workgroups still read when it is written."""

import ctypes

import pytest
import torch

# As in the other host checks: fake device pointers, so GPU-less hosts only.
if torch.cuda.device_count() > 0:
    pytest.skip("host checks run on GPU-less hosts", allow_module_level=True)

das = pytest.importorskip("paper_2609_34538_amd._lib")
SHAPE, HIP = -2, -6
POOL, LENS, NUM = 0x100000, 0x200000, 0x300000  # never dereferenced


def _call(len_out):
    c, b = das.DasCacheQ8C(), das.DasBatchC()
    base = c.base
    base.dtype, base.num_depths, base.num_layers, base.num_kv_heads, base.head_dim, base.num_pages = 1, 1, 1, 1, 64, 9
    base.num_k_planes, base.num_v_planes = 1, 1
    base.k_pool = base.v_pool = c.k_exp = c.v_exp = POOL
    b.batch, b.max_pages_per_seq, b.prefix_len, b.block_table = 5, 2, LENS, POOL
    return das.LIB.das_kv_append_q8(ctypes.byref(c), ctypes.byref(b), POOL, POOL, 8, NUM, len_out, None)


@pytest.mark.parametrize("at", [LENS, NUM])
@pytest.mark.parametrize("off", [-16, -4, 0, 4, 16])
def test_shared_elements_are_refused(at, off):
    assert _call(at + off) == SHAPE


@pytest.mark.parametrize("len_out", [LENS - 20, LENS + 20, NUM - 20, NUM + 20, None])
def test_neighbouring_arrays_are_not(len_out):
    """Five elements before or behind: such a call fails at its launch only, without a GPU."""
    assert _call(len_out) == HIP


def test_the_binding_reports_it():
    i32 = dict(dtype=torch.int32)
    cache = das.QuantCache.empty(1, 1, 9, 64, 1, {1: 0}, {1: 0}, device="cpu")
    batch = das.Batch(torch.zeros(3, **i32), torch.zeros((3, 2), **i32))
    new, n = torch.zeros((1, 1, 3, 4, 1, 64), dtype=torch.bfloat16), torch.zeros(3, **i32)
    call = das.PreparedAppendQ8(cache, batch, new, new, n, n)
    assert call._fn(*call._args, None) == SHAPE
