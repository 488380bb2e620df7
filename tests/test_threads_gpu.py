"""Two host threads that call one cache at once: attention over tables of their own and over chosen pages, on streams of their own
and on one."""
from concurrent.futures import ThreadPoolExecutor

import pytest
import torch

import four_bit as F
from test_cache_gpu import LENS, gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("streams", [1, 2])
def test_one_cache(streams):
    lens = LENS["ragged"](4, 4)
    cache = F.FourBit(nseq=4, Hq=16, Hkv=4, dh=64, dtype="bf16", page=32, cols=-(-int(lens.max()) // 32)).fill(lens, 2)
    dev, c = lens.cuda(), cache.c
    summary = c.summarise(c.new_summary(), dev)
    qs = [torch.randn(4, 16, 64, generator=gen(i)).bfloat16().cuda() for i in range(2)]
    tables = [c.select_pages(q, dev, summary, 7) for q in qs]
    want = [(c.attend(q, rows, table=table), c.attend_selected(q, dev, summary, 5)) for q, (table, rows) in zip(qs, tables)]
    assert not torch.equal(want[0][0][0], want[1][0][0]) and not torch.equal(tables[0][0], tables[1][0])
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(streams)]

    def run(i):
        with torch.cuda.stream(side[i % streams]):
            got = [(c.attend(qs[i], tables[i][1], table=tables[i][0]), c.attend_selected(qs[i], dev, summary, 5)) for _ in range(300)]
        side[i % streams].synchronize()
        return all(torch.equal(x, y) for g in got for a, b in zip(g, want[i]) for x, y in zip(a, b))

    with ThreadPoolExecutor(2) as pool:
        assert all(f.result() for f in [pool.submit(run, i) for i in range(2)])
