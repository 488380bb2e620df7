"""Two host threads that call one cache at once, on stand-ins for the library that take their time."""
import time
from concurrent.futures import ThreadPoolExecutor

import pytest
import torch

import stand_in
from paper_2502_03805_b200 import PageSummary


@pytest.fixture
def cache(monkeypatch):
    c = stand_in.cache(monkeypatch)
    c._ref = object()
    return c


Q, LENS = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 2, dtype=torch.int32)


def both(f, *arguments):
    with ThreadPoolExecutor(2) as pool:
        return [x.result() for x in [pool.submit(f, *a) for a in arguments]]


def test_tables_of_two_threads(cache):
    """The library reads a description some time after it was given its address."""
    seen = []

    def decode(handle, ref, q, strides, lens, out, lse, ws, size, raw):
        time.sleep(0.02)
        seen.append((out, ref._obj.page_table, ref._obj.max_pages))
        return 0
    cache._decode = decode
    tables = [torch.zeros(2, 2, 5, dtype=torch.int32) for _ in range(2)]
    outs = [torch.empty(2, 4, 64, dtype=torch.bfloat16) for _ in range(2)]
    cache.attend(Q, LENS, outs[0], table=tables[0])                 # the description is there already
    seen.clear()

    def attend(i):
        for _ in range(3):
            cache.attend(Q, LENS, outs[i], table=tables[i])
    both(attend, (0,), (1,))
    want = {out.data_ptr(): (t.data_ptr(), 5) for out, t in zip(outs, tables)}
    assert len(seen) == 6 and all(want[out] == (table, columns) for out, table, columns in seen)


def test_choices_of_two_threads_on_one_stream(cache):
    """A choice goes into tables that the stream's calls share: attention over it is enqueued before the next choice."""
    order = []

    def select(handle, ref, q, *rest):
        order.append(("choose", q))
        time.sleep(0.02)
        return 0

    def decode(handle, ref, q, *rest):
        order.append(("attend", q))
        return 0
    cache._select, cache._decode = select, decode
    summary = PageSummary(torch.zeros(9, 2, 64, dtype=torch.int8), torch.zeros(9))
    queries = [Q.clone() for _ in range(2)]

    def attend(q):
        for _ in range(3):
            cache.attend_selected(q, LENS, summary, 4)
    both(attend, (queries[0],), (queries[1],))
    assert len(order) == 12
    for (a, q), (b, r) in zip(order[::2], order[1::2]):
        assert (a, b) == ("choose", "attend") and q == r
