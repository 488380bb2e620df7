"""Numbers of rows and pages that are given as something else than an int, on stand-ins for the library: what is allocated and
what the library is told agree, also when a tensor has changed its value since the call before."""
import numpy as np
import pytest
import torch

import stand_in
from paper_2502_03805_b200 import PageSummary


@pytest.fixture
def cache(monkeypatch):
    return stand_in.cache(monkeypatch)


COUNTS = [lambda: 3, lambda: np.int64(3), lambda: torch.tensor(3), lambda: torch.tensor([3])]


@pytest.mark.parametrize("count", COUNTS)
def test_rows_loaded(cache, count):
    lens, n = torch.zeros(2, 2, dtype=torch.int32), count()
    for more in (0, 4, -5):
        n += more
        for out in cache.load(lens, n):
            assert out.shape == (2, 2, int(n), 64)
        given = [torch.empty(2, 2, int(n), 64, dtype=torch.bfloat16) for _ in range(2)]
        cache.load(lens, n, *given)
        assert cache.told[-2:] == [int(n), int(n)]
        with pytest.raises(ValueError):
            cache.load(lens, n + 1, *given)
    with pytest.raises(TypeError):
        cache.load(lens, 3.0)


@pytest.mark.parametrize("count", COUNTS)
def test_pages_chosen(cache, count):
    lens, q = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    summary = PageSummary(torch.zeros(9, 2, 64, dtype=torch.int8), torch.zeros(9))
    n = count()
    for more in (0, 4, -3):
        n += more
        table, rows = cache.select_pages(q, lens, summary, n)
        assert table.shape == (2, 2, int(n)) and cache.told[-1] == int(n)
        cache.attend_selected(q, lens, summary, n)
        assert cache.told[-1] == int(n) and cache._chosen[0, int(n)][0].shape == (2, 2, int(n))
        assert cache._parts[int(n)][0].max_pages == int(n)
    assert sorted(cache._chosen) == [(0, 3), (0, 4), (0, 7)]
    for call in (cache.select_pages, cache.attend_selected):
        with pytest.raises(TypeError):
            call(q, lens, summary, 4.0)
