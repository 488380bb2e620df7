"""What the errors of a choice of pages say, with the library's own refusals and without a GPU."""
import ctypes as C

import pytest
import torch

import stand_in
from paper_2502_03805_b200 import PageSummary
from paper_2502_03805_b200 import binding as B
from paper_2502_03805_b200 import build


@pytest.fixture
def cache(monkeypatch):
    build.build_library()
    c = stand_in.cache(monkeypatch)
    c._fake = C.create_string_buffer(4096)                 # no call comes as far as to use it
    c.handle, c._ref, c._select = C.addressof(c._fake), C.byref(c.desc), B.load().criticalkv_select_pages
    return c


@pytest.mark.parametrize("name", ["select_pages", "attend_selected"])
@pytest.mark.parametrize("pages,kw", [(1, {}), (2, dict(first=2)), (4, dict(first=0, last=5)), (4, dict(first=-1)), (4, dict(last=-2))])
def test_pages_that_do_not_hold_the_first_and_the_last(cache, name, pages, kw):
    q, lens = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 2, dtype=torch.int32)
    summary = PageSummary(torch.zeros(9, 2, 64, dtype=torch.int8), torch.zeros(9))
    with pytest.raises(B.CriticalKVError) as e:
        getattr(cache, name)(q, lens, summary, pages, **kw)
    assert e.value.status == B.CKV_EINVAL
    for part in (f"pages={pages}", f"first={kw.get('first', 1)}", f"last={kw.get('last', 1)}"):
        assert part in str(e.value)
