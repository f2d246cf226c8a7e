"""A 4-bit cache is made for the head dim that is asked for, or not at all."""

import pytest

das = pytest.importorskip("paper_2609_34538_amd._lib")


@pytest.mark.parametrize("head_dim", [64, 96, 128])
def test_head_dims(head_dim):
    assert das.Quant4Cache.empty(1, 2, 3, head_dim, 1, {1: 0}, {1: 0}, device="cpu").head_dim == head_dim


@pytest.mark.parametrize("head_dim", [16, 72, 80, 100, 127])
def test_head_dims_between_blocks(head_dim):
    with pytest.raises(ValueError, match="head_dim"):
        das.Quant4Cache.empty(1, 2, 3, head_dim, 1, {1: 0}, {1: 0}, device="cpu")
