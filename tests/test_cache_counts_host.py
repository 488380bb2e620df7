"""Numbers of rows and pages that are given as something else than an int, on stand-ins for the library: what is allocated and
what the library is told agree, also when a tensor has changed its value since the call before."""
import numpy as np
import pytest
import torch

from paper_2502_03805_b200 import PagedCache, PageSummary
from paper_2502_03805_b200 import binding as B
from paper_2502_03805_b200 import cache as cache_module


@pytest.fixture
def cache(monkeypatch):
    monkeypatch.setattr(cache_module, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(cache_module, "_current_device", lambda: 0)
    monkeypatch.setattr(cache_module, "_capturing", lambda: False)
    told = []
    c = PagedCache.__new__(PagedCache)
    c.nseq, c.Hq, c.Hkv, c.dh, c.num_pages, c.max_pages = 2, 4, 2, 64, 9, 8
    c.dtype, c.torch_dtype, c.device, c._index = "bf16", torch.bfloat16, torch.device("cpu"), 0
    c.desc = B.make_cache(nseq=2, Hq=4, Hkv=2, dh=64, dtype="bf16", format="plain", page_size=16, num_pages=9, max_pages=8,
                          k_pages=256, v_pages=256, page_table=256)
    c.handle, c._owned, c._ref, c._plans, c._seen = None, False, None, {}, {0}
    c._ws, c._ws_bytes, c._parts, c._chosen, c._out_shape = {}, 256, {}, {}, (2, 4, 64)
    c._out_like, c._lse_like = torch.empty(2, 4, 64, dtype=torch.bfloat16), torch.empty(2, 4)
    c._load = lambda handle, ref, lens, n, strides, how, K, V, raw: told.append(n) or 0
    c._select = lambda handle, ref, q, strides, lens, codes, scale, pages, *rest: told.append(pages) or 0
    c._decode = lambda *args: 0
    c.told = told
    return c


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
