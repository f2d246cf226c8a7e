"""The commit into the 4-bit cache and the way back refuse grids that HIP does not take, and no
smaller ones: both sides of the limit, before any HIP call."""

import ctypes

import pytest
import torch

# As in the other host checks: fake device pointers, so GPU-less hosts only.
if torch.cuda.device_count() > 0:
    pytest.skip("host-validation checks run on GPU-less hosts", allow_module_level=True)

das = pytest.importorskip("paper_2609_34538_amd._lib")
from test_draft_validation import _cache  # noqa: E402
from test_serve_validation import _batch  # noqa: E402

SHAPE, HIP = -2, -6  # HIP: past every check, to the launch that fails on this host
FAR = 1 << 48        # between arrays


@pytest.mark.parametrize("hkv,dh,planes,layers", [
    (1, 96, (2, 1), (2 ** 24 - 1) // 3),          # one workgroup a (plane, layer)
    (1, 128, (1, 1), (2 ** 24 - 1) // 2),
    (60, 64, (2, 1), (2 ** 24 - 1) // 30),        # ten
    (4, 96, (1, 2), (2 ** 24 - 1) // 3),          # twelve blocks: one
    (5, 96, (1, 2), (2 ** 24 - 1) // 6),          # fifteen: two
    (65535, 128, (1, 1), (2 ** 24 - 1) // 43690),
])
def test_both_sides_of_the_limit(hkv, dh, planes, layers):
    for more, status in ((0, HIP), (1, SHAPE)):
        c = _cache(num_kv_heads=hkv, head_dim=dh, num_layers=layers + more, num_k_planes=planes[0],
                   num_v_planes=planes[1], num_pages=1, k_pool=FAR, v_pool=2 * FAR, k_exp=3 * FAR, v_exp=4 * FAR)
        c.base.k_plane[4] = 0
        b = _batch()
        assert das.LIB.das_kv_append_q4(ctypes.byref(c), ctypes.byref(b), 5 * FAR, 6 * FAR, 1, 7 * FAR, None,
                                        None) == status
        assert das.LIB.das_kv_read_q4(ctypes.byref(c), ctypes.byref(b), 7 * FAR, 7 * FAR, 1, 5 * FAR, 6 * FAR,
                                      None) == status


def test_counts_at_the_ends_of_their_type():
    top = 2 ** 31 - 1
    for kw in (dict(num_layers=top), dict(num_layers=top, num_k_planes=top, num_v_planes=top),
               dict(num_layers=top, num_k_planes=top, num_v_planes=top, num_kv_heads=65535, head_dim=128)):
        c, b = _cache(**kw), _batch()
        assert das.LIB.das_kv_append_q4(ctypes.byref(c), ctypes.byref(b), FAR, 2 * FAR, 1, 3 * FAR, None, None) == SHAPE
        assert das.LIB.das_kv_read_q4(ctypes.byref(c), ctypes.byref(b), 3 * FAR, 3 * FAR, 1, FAR, 2 * FAR, None) == SHAPE
