"""The comparison of decode_bounds.py itself: mistakes planted in a result are seen."""
import math

import pytest
import torch

import decode_bounds as D


@pytest.fixture
def case():
    g = torch.Generator().manual_seed(1)
    kv, vv = (torch.randn(2, 16, 64, generator=g).double() for _ in range(2))
    q = torch.randn(1, 4, 64, generator=g) * 0.1
    table, lens = torch.tensor([[[0], [1]]], dtype=torch.int32), torch.tensor([[7, 0]], dtype=torch.int32)
    return D.decode(q, kv, vv, table, lens, 16, 0.125, "plain", "f32", "cuda"), lens


@pytest.mark.parametrize("what", ["none", "nan in out", "nan in lse", "+inf in lse", "row of an empty head", "11-bit weights"])
def test_planted_mistakes(case, what):
    want, lens = case
    out, lse = want[0].clone(), want[1].clone()
    if what == "nan in out":
        out[0, 1, 3] = math.nan
    elif what == "nan in lse":
        lse[0, 0] = math.nan
    elif what == "+inf in lse":
        lse[0, 3] = math.inf
    elif what == "row of an empty head":
        out[0, 2, 0] = 1e-30
    elif what == "11-bit weights":
        out[0, :2] *= 1 + 2.0 ** -12
    if what == "none":
        D.check((out, lse), want, lens, 2)
        return
    with pytest.raises(AssertionError):
        D.check((out, lse), want, lens, 2)
