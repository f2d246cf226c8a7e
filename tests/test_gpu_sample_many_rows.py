"""das_sample on more rows than the card has compute units, where a row has 512 threads:
filters, ties, lists around their bound, values outside the counted range, infinities."""

from __future__ import annotations

import pytest
import torch

from test_gpu_sample import _logits, check

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
B, W = 130, 2  # 260 rows

T = [1.0, 0.7, 1.5, 0.0, 0.9, 30.0, 0.05, 1.2, 1.0, 0.8]
K = [0, 20, 3, 5, 0, 1, 0, 2000, 700, 50]
P = [1.0, 1.0, 0.9, 0.5, 0.95, 0.3, 0.999, 0.7, 1.0, 0.99]
LOW = [0.0, 0.05, 0.0, 0.1, 0.02, 0.0, 0.0, 0.0, 1e-6, 0.3]
ALL = dict(T=T * 13, k=K * 13, p=P * 13, low=LOW * 13)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("kind", ["flat", "normal", "peaked"])
@pytest.mark.parametrize("V", [1, 513, 4099])
def test_filters(dtype, kind, V):
    check(*_logits(V, B, W, V, dtype, kind), **ALL)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("filt", [{}, dict(k=[40] * B), dict(p=[0.9] * B), dict(low=[0.05] * B), dict(T=[0.0] * B)],
                         ids=["none", "top_k", "top_p", "min_p", "greedy"])
def test_one_filter(dtype, filt):
    check(*_logits(3, B, W, 9001, dtype, "peaked"), **filt)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_equal_logits(dtype):
    z, u = _logits(2, B, W, 5000, dtype)
    z[:65] = 0.25
    z[65:] = torch.where(z[65:] > 1.0, 1.0, -1.0).to(dtype)
    check(z, u, **ALL)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("kept", [511, 512, 513])
def test_kept_tokens_around_the_bound_of_a_list(dtype, kept):
    """As for few rows: kept tokens at 210 and more, where bf16 rows are not counted by value."""
    z, u = _logits(7, B, W, 4000, dtype)
    g = torch.Generator(device=DEV).manual_seed(8)
    at = torch.randperm(4000, generator=g, device=DEV)[:kept]
    z[:, :, at] = (212 + torch.rand((B, W, kept), generator=g, device=DEV)).to(dtype)
    z[65:, :, at] = 210.0
    check(z, u, T=[1.0, 0.8] * 65, k=([kept] * 5 + [0] * 5) * 13, p=[0.9, 1.0, 0.7, 0.99, 1.0] * 26,
          low=[0.0, 0.01, 0.0, 0.2, 1.0] * 26)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_infinities_nan_and_the_lowest(dtype):
    z, u = _logits(3, B, W, 3001, dtype)
    z[0::5, :, ::2] = float("nan")
    z[1::5] = float("-inf")
    z[2::5, :, [5, 700, 2999]] = float("inf")
    z[3::5, :, 1:] = float("-inf")
    z[4::5, :, 10:] = torch.finfo(dtype).min
    check(z, u, **{**ALL, "T": [1.0, 0.5] * 65})
