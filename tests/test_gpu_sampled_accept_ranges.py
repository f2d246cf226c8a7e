"""Verification of drawn proposals at the ends of its numbers: tokens whose weight is nothing or
next to nothing under a low temperature, with random numbers of 0."""

from __future__ import annotations

import pytest
import torch

from test_gpu_sampled_accept import BF16, DEV, F32, I32, Call

pytestmark = pytest.mark.gpu


def _spread(seed, B, w, V, T, dtype):
    """Logits of some thousand temperatures' spread, none within 8 temperatures of where the
    64-bit exponential ends (745.1 below the largest), so that a sum's factor moves none over it."""
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn((B, w, V), generator=g) * 400 * T + 3).to(dtype)
    d = (z.max(-1, keepdim=True).values - z).double() / T
    z[(d > 737) & (d < 753)] = (3 - 3000 * T)
    return z


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [1e-3, 0.05])
@pytest.mark.parametrize("draft", [True, False])
def test_numbers_of_zero_at_low_temperatures(dtype, T, draft):
    """A draw of 0 is the first token that weighs anything, and a uniform of 0 accepts what p
    gives anything: not tokens whose exponential is 0."""
    B, w, V = 24, 4, 9000
    z, d = (_spread(s, B, w, V, T, dtype) for s in (1, 2))
    g = torch.Generator().manual_seed(5)
    # proposals with and without weight
    likely = torch.topk(z.float(), 40, -1).indices
    y = likely.gather(-1, torch.randint(0, 40, (B, w, 1), generator=g))[..., 0]
    y = torch.where(torch.rand((B, w), generator=g) < 0.7, y, torch.randint(0, V, (B, w), generator=g)).int().to(DEV)
    t, zeros = torch.full((B,), T, device=DEV), torch.zeros((B, w), device=DEV)
    z, d = z.to(DEV), d.to(DEV)
    for tested in (None, torch.zeros(B, **I32)):
        for u in (zeros, None):
            got = Call(z, d if draft else None, y, t, t if draft else None, tested, u=u, v=torch.zeros_like(t)).check()
            drawn = got["num_emitted"] > got["accepted"]
            assert drawn.sum() > B // 3
            if u is zeros and tested is None:
                assert 0 < got["accepted"].max() and got["accepted"].min() < w


@pytest.mark.parametrize("below", [690.0, 700.0, 730.0])
def test_a_token_of_hardly_any_weight_counts(below):
    """exp(-below) is no 0 in 64 bits: such a token is accepted at a uniform of 0 and drawn at
    a draw of 0, and one of exp(-750) is neither."""
    V, T = 600, 0.0625
    z = torch.full((2, 2, V), 8.0 - 900 * T, device=DEV)
    z[:, :, 500] = 8.0
    z[:, :, 100] = 8.0 - below * T
    z[:, :, 50] = 8.0 - 750 * T
    y = torch.tensor([[100, 50], [500, 50]], **I32)
    t, zeros = torch.full((2,), T, device=DEV), torch.zeros((2, 2), device=DEV)
    got = Call(z, None, y, t, u=zeros, v=torch.zeros_like(t)).check()
    assert got["accepted"].tolist() == [1, 1] and got["emitted"][:, 1].tolist() == [100, 100]
