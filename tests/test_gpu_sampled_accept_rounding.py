"""Verification of drawn proposals where a token's residual is under the rounding of the rows' sums."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from test_gpu_sampled_accept import DEV, I32, Call, reference

pytestmark = pytest.mark.gpu


def test_rounding_of_the_sums_leaves_no_token():
    """Token 0 is as likely to target and draft, to 2^-43 of it, at the logits where one row's sum
    came out too small and the other's too large by most when the largest logit's exponent was
    rounded by itself: their residual is nothing, and the first token that can be drawn is 1."""
    V = 8192
    z, d = (torch.empty((1, 1, V), device=DEV) for _ in range(2))
    z[...], d[...] = 5.091631889343262, 5.310670852661133
    z[..., 5], d[..., 5] = 5.1348748207092285, 5.6615376472473145
    z[..., 0], d[..., 0] = -0.20177435874938965, 0.019999993965029716
    z[..., -22:] = -float("inf")
    y, u, v = torch.full((1, 1), 5, **I32), torch.full((1, 1), 0.99, device=DEV), torch.zeros(1, device=DEV)
    f = lambda t: t[0].double().cpu().numpy()  # noqa: E731
    p, q = (np.exp(np.longdouble(f(x))[0]) for x in (z, d))
    assert -(2.0 ** -42) < p[0] / p.sum() / (q[0] / q.sum()) - 1 <= 0
    assert reference([5], f(z), [0.99], 0.0, f(d))[:2] == (0, [1])
    got = Call(z, d, y, u=u, v=v).check()
    assert got["emitted"][0, 0] == 1
