"""Choice of pages at the limits that the header states: 128 query heads a KV head, tables of 32768 pages, all of them held."""
import numpy as np
import pytest
import torch

from canary_util import Guarded
from paper_2502_03805_b200 import PagedCache, PageSummary
from paper_2502_03805_b200 import binding as B
from test_cache_gpu import gen

pytestmark = pytest.mark.gpu
PAGES, POOL, SIZE = 32768, 97, 16
LEAST = np.float32(2.0 ** -100)


def scores(q, codes, scales):
    """Of every page of the pool, the largest over the query heads [G, dh], by the documented rule."""
    x = q.float().numpy()
    scale = np.maximum(np.abs(x).max(-1) / np.float32(127), LEAST)
    code = np.clip(np.rint(x * (np.float32(1) / scale)[:, None]), -127, 127).astype(np.int64)
    c = codes.numpy().astype(np.int64)
    total = np.clip(code, 0, None) @ c[:, 0].T + np.clip(code, None, 0) @ c[:, 1].T           # [G, pool]: codes[0] >= codes[1]
    return ((total.astype(np.float32) * scale[:, None]) * scales.numpy()).max(0)


def check(c, table, held, score, call, count, first, last):
    chosen, pages, rows = (Guarded(s, torch.int32, fill=-9) for s in ((1, 1, count), (1, 1, count), (1, 1)))
    call(count, first=first, last=last, table=pages.t, rows=rows.t, chosen=chosen.t)
    j = np.arange(held)
    key = score[table.numpy()[0, 0, :held]]
    rank = np.lexsort((j, -key, ~((j < first) | (j >= held - last))))
    want = np.sort(rank[:count])
    rest = np.full(count - len(want), -1)
    assert np.array_equal(chosen.t.cpu().numpy()[0, 0], np.concatenate([want, rest]))
    assert np.array_equal(pages.t.cpu().numpy()[0, 0], np.concatenate([table.numpy()[0, 0, want], rest]))
    assert int(rows.t) == len(want) * SIZE - (5 if held - 1 in want else 0)
    assert chosen.intact() and pages.intact() and rows.intact() and c.device_status() == 0


@pytest.mark.parametrize("flags", [0, B.CKV_FLAG_SELECT_NO_CLUSTER])
@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 128), (torch.float32, 128), (torch.float32, 64)])
@pytest.mark.parametrize("equal", [False, True])
def test_the_largest_choice(flags, dtype, dh, equal):
    g = gen(dh)
    pool = torch.zeros(POOL, SIZE, dh, dtype=dtype, device="cuda")
    table = torch.randint(0, POOL, (1, 1, PAGES), generator=g, dtype=torch.int32)
    codes = torch.randint(-127, 128, (POOL, 2, dh), generator=g, dtype=torch.int32).to(torch.int8).sort(dim=1, descending=True).values
    scale = torch.rand(POOL, generator=g) + 0.5
    if equal:
        codes[:], scale[:] = codes[:1].clone(), scale[:1].clone()
    q = torch.randn(1, 128, dh, generator=g).to(dtype)
    name = "f32" if dtype == torch.float32 else "bf16"
    c = PagedCache(Hq=128, dtype=name, k_pages=pool, v_pages=pool.clone(), page_table=table.cuda(),
                   flags=flags | B.CKV_FLAG_DEBUG_CHECKS)
    summary, dev = PageSummary(codes.cuda(), scale.cuda()), q.cuda()
    score = scores(q[0], codes, scale)
    for held in (PAGES, PAGES - 1, 513):
        lens = torch.full((1, 1), held * SIZE - 5, dtype=torch.int32, device="cuda")
        call = lambda count, **kw: c.select_pages(dev, lens, summary, count, **kw)  # noqa: E731
        for count, first, last in ((1, 0, 0), (64, 1, 1), (1024, 0, 1024), (1025, 1000, 25), (5000, 7, 3), (held - 1, 1, 0), (held, 0, 1),
                                   (held + 3, 1, 1)):
            check(c, table, held, score, call, count, min(first, count), last)


def test_the_reference_scores_as_the_other_tests_do():
    from test_pages_gpu import choose
    g = gen(3)
    table = torch.randint(0, POOL, (1, 1, 60), generator=g, dtype=torch.int32)
    codes = torch.randint(-127, 128, (POOL, 2, 64), generator=g, dtype=torch.int32).to(torch.int8).sort(dim=1, descending=True).values
    scale = torch.rand(POOL, generator=g) + 0.5
    q = torch.randn(1, 3, 64, generator=g)
    want = choose(q, torch.tensor([[60 * SIZE - 5]]), codes.numpy(), scale.numpy(), table.numpy(), SIZE, 11, 1, 2)
    j, key = np.arange(60), scores(q[0], codes, scale)[table.numpy()[0, 0]]
    assert sorted(np.lexsort((j, -key, ~((j < 1) | (j >= 58))))[:11]) == want[0, 0]
