"""Summaries of pages, the choice of pages and attention over them: whole numbers equal to the plain form's, attention against
64 bits over the rows of the chosen pages."""
import math
from concurrent.futures import ThreadPoolExecutor

import numpy as np
import pytest
import torch

import cache_ref as R
import decode_bounds as D
import four_bit as F
from canary_util import Guarded
from paper_2502_03805_b200 import PagedCache, PageSummary, Rotary
from paper_2502_03805_b200 import binding as B
from paper_2502_03805_b200 import rope_frequencies
from test_cache_gpu import LENS, Cache, gen

pytestmark = pytest.mark.gpu
FORMATS = ["plain", "e4m3", "int8", "e2m1"]
LEAST = np.float32(2.0 ** -100)
MOVES = 16


def make(fmt, **kw):
    return F.FourBit(**kw) if fmt == "e2m1" else Cache(fmt=fmt, **kw)


def float32_keys(cache):
    """What the key pages stand for, as the float32 numbers that the library sees (code times scales, each step rounded)."""
    return cache.values()[0].float().numpy()          # one product of a code (times an exact group scale) and a scale


def summary_of(keys, rows):
    """codes [2, dh], scale of a page [page_size, dh] with `rows` rows."""
    x = keys[:rows]
    with np.errstate(invalid="ignore", over="ignore"):
        top = np.abs(x).max()
        scale = top / np.float32(127)
        scale = LEAST if scale < LEAST else np.float32(scale)
        if not np.isfinite(top):
            return np.zeros((2, x.shape[1]), np.int8), scale
        r = np.float32(1) / scale
        up, down = np.ceil(x.max(0) * r), np.floor(x.min(0) * r)
    return np.clip(np.stack([up, down]), -127, 127).astype(np.int8), scale


def choose(q, lens, codes, scales, table, page_size, count, first, last):
    """Chosen pages of every head by the documented rule, in numpy."""
    nseq, Hkv, _ = table.shape
    G = q.shape[1] // Hkv
    x = q.float().numpy()
    out = {}
    for s in range(nseq):
        for g in range(Hkv):
            held = -(-int(lens[s, g]) // page_size)
            if held <= count:
                out[s, g] = list(range(held))
                continue
            key = np.full(held, -np.inf)
            nan = np.zeros(held, bool)
            absent = np.zeros(held, bool)
            for h in range(g * G, (g + 1) * G):
                with np.errstate(invalid="ignore", over="ignore", under="ignore"):
                    top = np.abs(x[s, h]).max()
                    scale = top / np.float32(127)
                    scale = LEAST if scale < LEAST else np.float32(scale)
                    code = np.zeros(x.shape[2], np.int64)
                    if np.isfinite(top):
                        code = np.clip(np.rint(x[s, h] * (np.float32(1) / scale)), -127, 127).astype(np.int64)
                    for j in range(held):
                        p = int(table[s, g, j])
                        if not 0 <= p < codes.shape[0]:
                            absent[j] = True
                            continue
                        c = codes[p].astype(np.int64)
                        total = np.maximum(code * c[0], code * c[1]).sum()
                        f = np.float32(np.float32(total) * scale) * np.float32(scales[p])
                        nan[j] |= bool(np.isnan(f))
                        if not np.isnan(f):
                            key[j] = max(key[j], float(f))
            rank = sorted(range(held), key=lambda j: (not (j < first or j >= held - last), absent[j], not nan[j],
                                                      0.0 if nan[j] else -key[j], j))
            out[s, g] = sorted(rank[:count])
    return out


def check_choice(cache, q, lens, summary, count, first, last, c=None):
    c = cache.c if c is None else c
    nseq, Hkv = lens.shape
    table, rows, chosen = (Guarded(shape, torch.int32, fill=-9) for shape in ((nseq, Hkv, count), (nseq, Hkv), (nseq, Hkv, count)))
    got = c.select_pages(q.cuda(), lens.cuda(), summary, count, first=first, last=last, table=table.t, rows=rows.t, chosen=chosen.t)
    assert got[0] is table.t and got[1] is rows.t and table.intact() and rows.intact() and chosen.intact()
    now = cache.table_dev.cpu()
    want = choose(q, lens, summary.codes.cpu().numpy(), summary.scale.cpu().numpy(), now.numpy(), cache.page, count, first, last)
    for (s, g), pages in want.items():
        n = len(pages)
        assert chosen.t[s, g].cpu().tolist() == pages + [-1] * (count - n)
        assert table.t[s, g].cpu().tolist() == now[s, g][torch.tensor(pages, dtype=torch.long)].tolist() + [-1] * (count - n)
        held = -(-int(lens[s, g]) // cache.page)
        assert int(rows.t[s, g]) == n * cache.page - (held * cache.page - int(lens[s, g]) if held - 1 in pages else 0)
    return want, table.t, rows.t


def check_attention(cache, q, want, lens, got, rows, c=None):
    """Attention over the rows of the chosen pages: a table of these pages in 64 bits."""
    nseq, Hkv = lens.shape
    cols = max([len(p) for p in want.values()] + [1])
    table = torch.zeros((nseq, Hkv, cols), dtype=torch.int32)
    for (s, g), pages in want.items():
        table[s, g, :len(pages)] = cache.table[s, g][torch.tensor(pages, dtype=torch.long)]
    scale = 1.0 / math.sqrt(cache.dh)
    if cache.fmt == "e2m1":
        exact = F.attention(q, cache, rows.cpu(), scale, "tensor", table)
    else:
        exact = D.decode(q, *cache.values(), table, rows.cpu(), cache.page, scale, cache.fmt, cache.dtype,
                         "tensor" if cache.dtype == "bf16" else "cuda", cache.vs, MOVES)
    D.check(got, exact, rows.cpu(), q.shape[1] // Hkv)


# ---- summaries -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh,page,nseq,Hkv,lens", [(128, 64, 1, 2, "ragged"), (64, 16, 3, 2, "edges"), (64, 256, 1, 3, "ragged"),
                                                   (128, 32, 2, 1, "short"), (128, 128, 40, 8, "edges")])
def test_summaries_bit_for_bit(dtype, fmt, dh, page, nseq, Hkv, lens):
    lens = LENS[lens](nseq, Hkv)
    cols = max(1, -(-int(lens.max()) // page))
    cache = make(fmt, nseq=nseq, Hq=Hkv, Hkv=Hkv, dh=dh, dtype=dtype, page=page, cols=cols, seed=dh).fill(lens, 5)
    n = cache.k.shape[0]
    codes, scale = Guarded((n, 2, dh), torch.int8, fill=99), Guarded((n,), torch.float32, fill=-1.0)
    summary = PageSummary(codes.t, scale.t)
    cache.c.summarise(summary, lens.cuda())
    keys = float32_keys(cache)
    want_codes, want_scale = np.full((n, 2, dh), 99, np.int8), np.full(n, -1.0, np.float32)
    for s in range(nseq):
        for g in range(Hkv):
            for j in range(-(-int(lens[s, g]) // page)):
                p = int(cache.table[s, g, j])
                want_codes[p], want_scale[p] = summary_of(keys[p], min(page, int(lens[s, g]) - j * page))
    assert np.array_equal(scale.t.cpu().numpy(), want_scale) and np.array_equal(codes.t.cpu().numpy(), want_codes)
    assert codes.intact() and scale.intact() and cache.c.device_status() == 0
    # only the pages with new rows
    start = (lens - torch.randint(0, 3 * page, lens.shape, generator=gen(7))).clamp(min=0).to(torch.int32)
    codes.t.fill_(99)
    scale.t.fill_(-1.0)
    cache.c.summarise(summary, lens.cuda(), start.cuda())
    for s in range(nseq):
        for g in range(Hkv):
            for j in range(cols):
                if j * page < int(lens[s, g]) and (j < int(start[s, g]) // page or start[s, g] == lens[s, g]):
                    p = int(cache.table[s, g, j])
                    want_codes[p], want_scale[p] = 99, -1.0
    assert np.array_equal(scale.t.cpu().numpy(), want_scale) and np.array_equal(codes.t.cpu().numpy(), want_codes)


def test_summaries_of_special_pages_wild_lengths_and_absent_pages():
    cache = make("plain", nseq=1, Hq=4, Hkv=4, dh=64, dtype="f32", page=16, cols=2, flags=B.CKV_FLAG_DEBUG_CHECKS)
    lens = torch.tensor([[32, 32, 32, 20]], dtype=torch.int32)
    cache.fill(lens, 3)
    pages = cache.table[0].long()
    cache.k[int(pages[0, 0])] = 0.0
    cache.k[int(pages[1, 0]), 3, 5] = math.inf
    cache.k[int(pages[1, 1]), 15, 63] = math.nan
    cache.k[int(pages[2, 0])] = 3.4028234e38
    cache.k[int(pages[2, 1]), 1:] = -1e-40
    summary = cache.c.new_summary()
    cache.c.summarise(summary, lens.cuda())
    assert cache.c.device_status() == 0
    for g in range(4):
        for j in range(2):
            p = int(pages[g, j])
            codes, scale = summary_of(cache.k[p].cpu().numpy(), min(16, int(lens[0, g]) - 16 * j))
            assert np.array_equal(summary.codes[p].cpu().numpy(), codes)
            assert float(summary.scale[p]) == float(scale) or (np.isnan(scale) and math.isnan(float(summary.scale[p])))
    again = cache.c.new_summary()
    cache.table_dev[0, 0, 1], cache.table_dev[0, 1, 0] = -1, cache.k.shape[0]
    cache.c.summarise(again, torch.tensor([[32, 2 ** 31 - 1, -4, 20]], dtype=torch.int32, device="cuda"),
                      torch.tensor([[-7, 0, 0, 40]], dtype=torch.int32, device="cuda"))
    assert cache.c.device_status() == B.CKV_EBOUNDS
    kept = [int(pages[0, 0]), int(pages[1, 1])]
    assert torch.equal(again.codes[kept], summary.codes[kept])
    rest = [p for p in range(cache.k.shape[0]) if p not in kept]
    assert not bool(again.codes[rest].any()) and not bool(again.scale[rest].any())


# ---- choice and attention --------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh,G,Hkv,nseq,page,lens,count,first,last", [
    (128, 4, 2, 1, 16, [[5000, 777]], 24, 1, 1), (64, 1, 3, 2, 32, [[900, 0, 33], [1, 32, 1500]], 7, 0, 2),
    (64, 9, 1, 2, 16, [[1025], [2000]], 40, 3, 0), (128, 16, 1, 1, 64, [[6553]], 10, 0, 0), (64, 40, 1, 1, 16, [[555]], 5, 2, 3),
    (128, 8, 8, 3, 128, [[300 * (i + 1) + j for i in range(8)] for j in (0, 3, 128)], 4, 1, 1), (64, 2, 2, 1, 16, [[4, 3]], 300, 1, 1)])
def test_choice_and_attention(dtype, fmt, dh, G, Hkv, nseq, page, lens, count, first, last):
    lens = torch.tensor(lens, dtype=torch.int32)
    cols = max(1, -(-int(lens.max()) // page))
    cache = make(fmt, nseq=nseq, Hq=G * Hkv, Hkv=Hkv, dh=dh, dtype=dtype, page=page, cols=cols, seed=dh + G).fill(lens, G)
    q = torch.randn(nseq, G * Hkv, dh, generator=gen(G + 1)).to(R.DT[dtype])
    summary = cache.c.summarise(cache.c.new_summary(), lens.cuda())
    want, table, rows = check_choice(cache, q, lens, summary, count, first, last)
    got = cache.c.attend(q.cuda(), rows, table=table)
    check_attention(cache, q, want, lens, got, rows)
    both = cache.c.attend_selected(q.cuda(), lens.cuda(), summary, count, first=first, last=last)
    assert torch.equal(both[0], got[0]) and torch.equal(both[1], got[1])
    full = cache.c.attend(q.cuda(), lens.cuda())                              # every page chosen: attention over all rows
    every = cache.c.attend_selected(q.cuda(), lens.cuda(), summary, max(cols, 2))
    assert torch.equal(every[0], full[0]) and torch.equal(every[1], full[1])
    assert cache.c.device_status() == 0 and cache.intact()


def test_without_clusters_and_on_many_heads_the_same_pages():
    for nseq, Hkv in ((1, 2), (50, 8)):
        lens = LENS["ragged"](nseq, Hkv)
        cache = make("e4m3", nseq=nseq, Hq=2 * Hkv, Hkv=Hkv, dh=64, dtype="bf16", page=16, cols=-(-int(lens.max()) // 16)).fill(lens, 2)
        q = torch.randn(nseq, 2 * Hkv, 64, generator=gen(3)).bfloat16()
        summary = cache.c.summarise(cache.c.new_summary(), lens.cuda())
        check_choice(cache, q, lens, summary, 6, 1, 1)
        apart = PagedCache(Hq=2 * Hkv, dtype="bf16", format="e4m3", k_pages=cache.k, v_pages=cache.v, k_scale=cache.ks,
                           v_scale=cache.vs, page_table=cache.table_dev, flags=B.CKV_FLAG_SELECT_NO_CLUSTER)
        check_choice(cache, q, lens, summary, 6, 1, 1, apart)


@pytest.mark.parametrize("cols", [3000, 20000])
def test_many_pages_with_equal_and_special_scores(cols):
    """Summaries made up: equal scores (the lower page wins), NaN (first), page ids outside the pool (last), scores of zero."""
    g = gen(4)
    n, dh = 97, 64
    pages = torch.zeros(n, 16, dh, dtype=torch.bfloat16, device="cuda")
    table = torch.randint(0, n, (1, 2, cols), generator=g, dtype=torch.int32)
    table[0, 0, 5], table[0, 0, 700], table[0, 1, cols // 2] = -3, n, 2 ** 31 - 1
    c = PagedCache(Hq=4, dtype="bf16", k_pages=pages, v_pages=pages.clone(), page_table=table.cuda())
    codes = torch.randint(-3, 4, (n, 2, dh), generator=g, dtype=torch.int8).sort(dim=1, descending=True).values
    scale = torch.ones(n)
    codes[7], scale[7] = 0, math.nan
    codes[11], scale[11] = 0, math.inf
    codes[12] = 0
    summary = PageSummary(codes.cuda(), scale.cuda())

    class Told:
        page, table_dev = 16, table
    told = Told()
    told.c = c
    for q in (torch.randint(-2, 3, (1, 4, dh), generator=g).bfloat16(), torch.zeros(1, 4, dh, dtype=torch.bfloat16)):
        for lens in ([[16 * cols, 16 * cols - 5]], [[16 * 1000 - 15, 17]]):
            for count, first, last in ((1, 0, 0), (64, 1, 1), (999, 3, 500), (2500, 0, 7)):
                check_choice(told, q, torch.tensor(lens, dtype=torch.int32), summary, count, first, last)
    q = torch.randn(1, 4, dh, generator=g).bfloat16()
    q[0, 1, 3], q[0, 2, 9] = math.nan, math.inf                               # of both heads: every page scores NaN
    check_choice(told, q, torch.tensor([[16 * cols, 500]], dtype=torch.int32), summary, 20, 2, 1)


@pytest.mark.parametrize("n", [2, 3, 40, 1500])
def test_borders_at_both_ends_of_the_order_of_scores(n):
    """Few pages, of which some score NaN, infinity, zero or minus infinity: the border is in the first or last of the bins that
    the scores are spread over."""
    dh = 64
    pages = torch.zeros(8, 16, dh, dtype=torch.bfloat16, device="cuda")
    codes, scale = torch.zeros(8, 2, dh, dtype=torch.int8), torch.ones(8)
    codes[0], codes[1], codes[2], codes[3] = 5, -5, 1, 2
    codes[4], codes[5] = 127, -127
    scale[4], scale[5], scale[7] = 3e38, 3e38, math.nan
    summary = PageSummary(codes.cuda(), scale.cuda())
    q = torch.full((1, 1, dh), 2.0, dtype=torch.bfloat16)

    class Told:
        page = 16
    told = Told()
    for seed in range(6):
        told.table_dev = torch.randint(-1 if seed % 2 else 0, 8, (1, 1, n), generator=gen(seed), dtype=torch.int32)
        told.c = PagedCache(Hq=1, dtype="bf16", k_pages=pages, v_pages=pages.clone(), page_table=told.table_dev.cuda())
        for count in sorted({1, n // 2 or 1, n - 1}):
            check_choice(told, q, torch.tensor([[16 * n - 3]], dtype=torch.int32), summary, count, 0, 0)


def test_scores_bound_the_logits():
    """The page with the largest logit of a single query is chosen when its bound stands out; and no page's best logit is
    above its score by more than the codes round."""
    lens = torch.tensor([[4000]], dtype=torch.int32)
    cache = make("plain", nseq=1, Hq=1, Hkv=1, dh=64, dtype="f32", page=16, cols=250).fill(lens, 3, spread=0.0)
    q = torch.randn(1, 1, 64, generator=gen(5))
    page, slot = int(cache.table[0, 0, 123]), 9
    cache.k[page, slot] = 3.0 * q[0, 0].cuda()
    summary = cache.c.summarise(cache.c.new_summary(), lens.cuda())
    chosen = torch.empty(1, 1, 1, dtype=torch.int32, device="cuda")
    cache.c.select_pages(q.cuda(), lens.cuda(), summary, 1, first=0, last=0, chosen=chosen)
    assert int(chosen) == 123
    keys = cache.values()[0]
    for j in range(250):
        p = int(cache.table[0, 0, j])
        bound = torch.maximum(q[0, 0].double() * summary.codes[p, 0].cpu().double(), q[0, 0].double() * summary.codes[p, 1].cpu().double())
        bound = bound.sum() * float(summary.scale[p])
        best = (keys[p] @ q[0, 0].double()).max()
        # codes are rounded outwards; the two float32 roundings in front of that and of the scale can undo 2^-22 of a value
        assert float(best) <= float(bound) + 2.0 ** -21 * float(q.abs().sum() * keys[p].abs().max())


def test_a_decode_loop_on_streams_and_in_a_graph():
    """Append, summarise the last pages, attend to chosen pages: eagerly, on another stream, and captured; the same bits."""
    nseq, Hq, Hkv, dh, rows = 2, 8, 2, 128, 700
    g = gen(6)
    rotary = Rotary(dh=dh, frequencies=rope_frequencies(dh), device="cuda:0")
    K, V = (torch.randn(nseq, Hkv, rows, dh, generator=g).bfloat16().cuda() for _ in range(2))
    steps = [tuple(torch.randn(nseq, h, 1, dh, generator=g).bfloat16().cuda() for h in (Hq, Hkv, Hkv)) for _ in range(5)]
    positions = [torch.full((nseq, 1), 9000 + i, dtype=torch.int32, device="cuda") for i in range(5)]

    def fresh():
        cache = PagedCache.allocate(nseq=nseq, Hq=Hq, Hkv=Hkv, dh=dh, dtype="bf16", rows=rows + 8, format="e2m1", page_size=16)
        lens = cache.store(K, V, cache.new_lengths())
        return cache, lens, cache.summarise(cache.new_summary(), lens)

    def step(cache, lens, summary, i, stream=None):
        q, k, v = steps[i]
        q, new = cache.append(q, k, v, positions[i], rotary, lens, stream=stream)
        cache.summarise(summary, new, lens, stream=stream)
        out = cache.attend_selected(q[:, :, 0], new, summary, 8, stream=stream)
        return out, new

    def loop(stream=None):
        cache, lens, summary = fresh()
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        outs = []
        for i in range(5):
            out, lens = step(cache, lens, summary, i, stream)
            outs.append(out)
        return outs, lens, summary, cache

    want, lens, summary, _ = loop()
    assert torch.equal(lens.cpu(), torch.full((nseq, Hkv), rows + 5, dtype=torch.int32))
    side = torch.cuda.Stream()
    other, _, summary2, cache2 = loop(side)
    side.synchronize()
    assert all(torch.equal(a, b) for x, y in zip(want, other) for a, b in zip(x, y))
    assert torch.equal(summary.codes, summary2.codes) and cache2.device_status() == 0

    cache, lens0, summary3 = fresh()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lens, outs = lens0, []
        for i in range(5):
            out, lens = step(cache, lens, summary3, i)
            outs.append(out)
    for _ in range(2):                      # replayed: the rows are written again, the same way
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(want, outs) for a, b in zip(x, y))
    eager = cache.attend_selected(steps[0][0][:, :, 0], lens, summary3, 8)    # its own buffers next to the graph's
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for x, y in zip(want, outs) for a, b in zip(x, y)) and bool(torch.isfinite(eager[0]).all())


def test_refusals():
    cache = PagedCache.allocate(nseq=2, Hq=4, Hkv=2, dh=64, dtype="bf16", rows=50, page_size=16)
    lens, summary = cache.new_lengths(), cache.new_summary()
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    for bad in (dict(lens=lens.long()), dict(lens=lens[:1]), dict(start=lens.cpu()), dict(summary=PageSummary(summary.codes[:1], summary.scale)),
                dict(summary=PageSummary(summary.codes, summary.scale.double())), dict(summary=PageSummary(summary.codes.cpu(), summary.scale))):
        with pytest.raises(ValueError):
            cache.summarise(**{**dict(summary=summary, lens=lens), **bad})
    ok = dict(q=q, lens=lens, summary=summary, pages=2)
    cache.select_pages(**ok)
    for bad in (dict(q=q.float()), dict(q=q[:, :2]), dict(lens=lens.long()), dict(table=torch.zeros(2, 2, 3, **i32)),
                dict(rows=torch.zeros(2, 1, **i32)), dict(chosen=torch.zeros(2, 2, 2, device="cuda")),
                dict(summary=PageSummary(summary.codes.transpose(0, 1), summary.scale))):
        with pytest.raises(ValueError):
            cache.select_pages(**{**ok, **bad})
    for bad in (dict(pages=1), dict(first=2), dict(first=-1), dict(last=3, first=0), dict(rows=lens)):
        with pytest.raises(B.CriticalKVError):
            cache.select_pages(**{**ok, **bad})
    for table in (torch.zeros(2, 2, **i32), torch.zeros(2, 2, 0, **i32), torch.zeros(2, 1, 3, **i32), torch.zeros(2, 2, 3, device="cuda")):
        with pytest.raises(ValueError):
            cache.attend(q, lens, table=table)
    out, lse = cache.attend_selected(q, lens, summary, 2)                     # empty heads
    assert not bool(out.any()) and bool((lse == -math.inf).all())


def test_wild_lengths_absent_pages_and_no_sequences():
    """Lengths outside the table are clipped, pages outside the pool score last and are treated as absent by attention."""
    lens = torch.tensor([[160, 160, 0]], dtype=torch.int32)
    cache = make("e2m1", nseq=1, Hq=6, Hkv=3, dh=64, dtype="bf16", page=16, cols=10, flags=B.CKV_FLAG_DEBUG_CHECKS).fill(lens, 3)
    summary = cache.c.summarise(cache.c.new_summary(), lens.cuda())
    q = torch.randn(1, 6, 64, generator=gen(2)).bfloat16()
    assert cache.c.device_status() == 0
    want, table, rows = check_choice(cache, q, lens, summary, 4, 1, 1)
    given = torch.tensor([[2 ** 31 - 1, 161, -2 ** 31]], dtype=torch.int32)
    got = cache.c.select_pages(q.cuda(), given.cuda(), summary, 4)
    assert cache.c.device_status() == B.CKV_EBOUNDS
    assert torch.equal(got[0], table) and torch.equal(got[1], rows)
    cache.table_dev[0, 0, 3:9] = torch.tensor([-1, cache.k.shape[0], 2 ** 31 - 1, -2 ** 31, -7, 10 ** 9], dtype=torch.int32, device="cuda")
    want, table, rows = check_choice(cache, q, lens, summary, 4, 1, 1)
    assert want[0, 0] == [0, 1, 2, 9] and cache.c.device_status() == B.CKV_EBOUNDS
    out, lse = cache.c.attend_selected(q.cuda(), lens.cuda(), summary, 7)              # three absent pages among the chosen
    want, table, rows = check_choice(cache, q, lens, summary, 7, 1, 1)
    there = [j for j in want[0, 0] if 0 <= int(cache.table_dev[0, 0, j]) < cache.k.shape[0]]
    only = {(0, 0): there, (0, 1): want[0, 1], (0, 2): []}
    check_attention(cache, q, only, lens, (out, lse), torch.tensor([[16 * len(there), 16 * 7, 0]], dtype=torch.int32))
    none = PagedCache(Hq=6, dtype="bf16", format="e2m1", k_pages=cache.k, v_pages=cache.v, k_scale=cache.ks, v_scale=cache.vs,
                      k_group_scale=cache.kg, v_group_scale=cache.vg, page_table=cache.table_dev[:0])
    empty = none.new_lengths()
    x = torch.zeros(0, 6, 64, dtype=torch.bfloat16, device="cuda")
    none.summarise(summary, empty)
    assert none.attend_selected(x, empty, summary, 4)[0].shape == (0, 6, 64)
    rotary = Rotary(dh=64, frequencies=rope_frequencies(64), device="cuda:0")
    assert none.append(x[:, :, None], x[:, :3, None], x[:, :3, None], torch.zeros(0, 1, dtype=torch.int32, device="cuda"), rotary,
                       empty)[0].shape == (0, 6, 1, 64)


def test_two_streams_at_once():
    """The same cache chooses and attends on two streams that run side by side, with other queries on each."""
    lens = LENS["ragged"](4, 4)
    cache = make("e2m1", nseq=4, Hq=16, Hkv=4, dh=128, dtype="bf16", page=32, cols=-(-int(lens.max()) // 32)).fill(lens, 2)
    qs = [torch.randn(4, 16, 128, generator=gen(i)).bfloat16().cuda() for i in range(2)]
    dev = lens.cuda()
    summary = cache.c.summarise(cache.c.new_summary(), dev)
    want = [[x.clone() for x in cache.c.attend_selected(q, dev, summary, pages)] for q, pages in zip(qs, (5, 5))]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(30):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(cache.c.attend_selected(qs[i], dev, summary, 5))
    torch.cuda.synchronize()
    for i in range(2):
        for out, lse in got[i]:
            assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])


def test_pages_behind_two_gigabytes():
    """A pool whose last pages lie more than 2^31 bytes behind its first: rows in, out, summarised, chosen and attended to."""
    n, page, dh, Hkv, Hq, rows = 2_200_000, 16, 128, 2, 8, 330
    k, v = (torch.empty((n, page, dh // 2), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.empty((n, page), device="cuda") for _ in range(2))
    kg, vg = (torch.empty((n, page, dh // 16), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    cols = -(-(rows + 1) // page)
    table = (n - 1 - torch.arange(Hkv * cols, dtype=torch.int32)).view(1, Hkv, cols).cuda()
    far = PagedCache(Hq=Hq, dtype="bf16", format="e2m1", k_pages=k, v_pages=v, k_scale=ks, v_scale=vs, k_group_scale=kg,
                     v_group_scale=vg, page_table=table)
    near = PagedCache.allocate(nseq=1, Hq=Hq, Hkv=Hkv, dh=dh, dtype="bf16", rows=rows + 1, format="e2m1", page_size=page)
    g = gen(8)
    K, V = (torch.randn(1, Hkv, rows, dh, generator=g).bfloat16().cuda() for _ in range(2))
    q, k1, v1 = (torch.randn(1, h, 1, dh, generator=g).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
    rotary = Rotary(dh=dh, frequencies=rope_frequencies(dh), device="cuda:0")
    pos = torch.full((1, 1), 9, dtype=torch.int32, device="cuda")
    results = []
    for c in (far, near):
        lens = c.store(K, V, c.new_lengths())
        summary = PageSummary(torch.empty((c.num_pages, 2, dh), dtype=torch.int8, device="cuda"), torch.empty(c.num_pages, device="cuda"))
        qr, lens = c.append(q, k1, v1, pos, rotary, lens)
        c.summarise(summary, lens)
        ids = c.page_table.long()
        results.append((qr, lens, *c.load(lens, rows + 1), summary.codes[ids], summary.scale[ids], *c.attend(qr[:, :, 0], lens),
                        *c.attend_selected(qr[:, :, 0], lens, summary, 6)))
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_two_threads_with_tables_of_other_lengths():
    """Caches of two host threads, each with a handle of its own, whose choices take different amounts of shared memory."""
    work = []
    for cols, pages in ((32768, 40), (12500, 17)):
        lens = torch.tensor([[16 * 100 + 3]], dtype=torch.int32)
        cache = make("plain", nseq=1, Hq=4, Hkv=1, dh=64, dtype="bf16", page=16, cols=101).fill(lens, cols)
        table = torch.full((1, 1, cols), -1, dtype=torch.int32, device="cuda")
        table[:, :, :101] = cache.table_dev
        wide = PagedCache(Hq=4, dtype="bf16", k_pages=cache.k, v_pages=cache.v, page_table=table)
        q, dev = torch.randn(1, 4, 64, generator=gen(cols)).bfloat16().cuda(), lens.cuda()
        summary = wide.summarise(wide.new_summary(), dev)
        want, rows = cache.c.select_pages(q, dev, summary, pages)
        work.append((wide, q, dev, summary, pages, want, rows))
    torch.cuda.synchronize()

    def choose(cache, q, dev, summary, pages, want, rows):
        with torch.cuda.stream(torch.cuda.Stream()):
            got = [cache.select_pages(q, dev, summary, pages) for _ in range(2000)]
            return all(torch.equal(t, want) and torch.equal(n, rows) for t, n in got[::100])

    with ThreadPoolExecutor(2) as pool:
        assert all(f.result() for f in [pool.submit(choose, *w) for w in work])
