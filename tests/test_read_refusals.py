"""A run of the cache that begins in front of its first key is refused by the binding (no GPU): the last keys are first=None, which the C call's -1 must not stand for here."""
import pytest
import torch

import paper_2409_16997_amd as ifa
from paper_2409_16997_amd import binding


@pytest.mark.parametrize("count", [None, 1, 9])
@pytest.mark.parametrize("first", [-1, -2, -(1 << 40)])
def test_no_first_below_zero(monkeypatch, first, count):
    reached = []
    monkeypatch.setattr(binding, "_native", type("Native", (), {"read": staticmethod(lambda *a: reached.append(a))}))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    cache = torch.zeros(1, 2, 9, 32, dtype=torch.uint8), torch.ones(1, 2, 9), torch.zeros(1, 2, 9, 32, dtype=torch.uint8), torch.ones(1, 2, 9)
    with pytest.raises(ifa.IntfaError, match="from -"):
        ifa.read_keys(*cache, first=first, count=count)
    assert not reached
