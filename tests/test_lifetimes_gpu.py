"""Memory that objects keep for themselves: not handed out again while a call that uses it is in flight on another stream,
and not shared by calls that run at the same time."""
import gc

import pytest
import torch

from paper_2502_03805_b200 import ChunkedPrefillCompressor, PagedCache, Rotary, rope_frequencies
from paper_2502_03805_b200 import binding as B

pytestmark = pytest.mark.gpu
HOLD = 2_000_000_000      # about a second: longer than a collection of Python's garbage takes


def gen(seed):
    return torch.Generator().manual_seed(seed)


def filled(rows, nseq=1, Hq=8, Hkv=2, dh=128, handle=None):
    g = gen(3)
    cache = PagedCache.allocate(nseq=nseq, Hq=Hq, Hkv=Hkv, dh=dh, dtype="bf16", rows=rows, handle=handle)
    K, V = (torch.randn(nseq, Hkv, rows, dh, generator=g).bfloat16().cuda() for _ in range(2))
    return cache, cache.store(K, V, cache.new_lengths())


@pytest.fixture
def handle():
    h = B.criticalkv_create(0)        # shared: an object's own handle waits for the GPU when it goes
    yield h
    torch.cuda.synchronize()
    B.criticalkv_destroy(h)


def handed_out_again(sizes, old, side):
    """Whether new blocks of these sizes are among the old ones, which `side` has not come to yet."""
    new = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    assert not side.query()
    return any(x.data_ptr() in old for x in new)


def test_a_rotary_dropped_while_it_runs(handle):
    q = torch.randn(1, 2, 3, 64, generator=gen(1)).cuda()
    pos = torch.zeros(1, 3, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    r = Rotary(dh=64, frequencies=rope_frequencies(64), device="cuda:0", handle=handle)
    at, size = {r.freq.data_ptr()}, r.freq.numel() * 8
    r.rotate(q, None, pos)                             # a kernel's first launch may wait for the GPU
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(HOLD)
        out, _ = r.rotate(q, None, pos)
    del r
    gc.collect()
    assert not handed_out_again([size] * 3, at, side)
    side.synchronize()
    assert torch.equal(out, q)                         # position 0


@pytest.mark.parametrize("as_argument", [False, True])
def test_a_cache_dropped_while_it_runs(handle, as_argument):
    cache, lens = filled(40000, handle=handle)
    q = torch.randn(1, 8, 128, generator=gen(1)).bfloat16().cuda()
    want = cache.attend(q, lens)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(HOLD)
        got = None if as_argument else cache.attend(q, lens)
    if as_argument:
        got = cache.attend(q, lens, stream=side)
    kept = [cache.k_pages, cache.v_pages, cache.page_table, *cache._ws.values()]
    at, sizes = {x.data_ptr() for x in kept[:3] + kept[4:]}, [x.numel() * x.element_size() for x in kept]
    assert len(kept) == 5                              # the workspaces of two streams
    del kept, cache
    gc.collect()
    assert not handed_out_again(sizes, at, side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_rows_that_the_next_step_drops():
    """(Uniform budgets: with adaptive ones to_cache uploads a list, for which the host waits.)"""
    g = gen(4)
    Hq, Hkv, dh, dm, w, n = 4, 2, 64, 64, 8, 900
    ch = ChunkedPrefillCompressor(Hq=Hq, Hkv=Hkv, dh=dh, dm=dm, w=w, pool_k=3, dtype="bf16", budget_mode="uniform")
    ch.step(*(torch.randn(*s, generator=g).bfloat16().cuda() for s in ((Hq, w, dh), (Hkv, n, dh), (Hkv, n, dh), (Hq, dh, dm))), 400)
    cache = PagedCache.allocate(nseq=1, Hq=Hq, Hkv=Hkv, dh=dh, dtype="bf16", rows=n)
    want = ch.K.clone()
    at, sizes = {x.data_ptr() for x in (ch.K, ch.V)}, [x.numel() * 2 for x in (ch.K, ch.V)]
    ch.to_cache(PagedCache.allocate(nseq=1, Hq=Hq, Hkv=Hkv, dh=dh, dtype="bf16", rows=n))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(HOLD)
    lens = ch.to_cache(cache, stream=side)
    ch.K = ch.V = None
    gc.collect()
    assert not handed_out_again(sizes, at, side)
    side.synchronize()
    K, _ = cache.load(lens, 400)
    assert torch.equal(K[0], want)


def test_two_streams_and_two_graphs_at_once_without_workspace_arguments():
    cache, lens = filled(30000)
    qs = [torch.randn(1, 8, 128, generator=gen(i)).bfloat16().cuda() for i in range(4)]
    want = [cache.attend(q, lens) for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    graphs, outs = [], []
    torch.cuda.synchronize()
    for q in qs[2:]:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(cache.attend(q, lens))
        graphs.append(graph)
    known = len(cache._ws)
    assert cache.workspace().data_ptr() == cache.workspace().data_ptr() != cache.workspace(streams[0]).data_ptr()
    assert len(cache._ws) == known + 1                 # the captures left none behind
    got = []
    for _ in range(20):
        got.append([cache.attend(q, lens, stream=s) for q, s in zip(qs[:2], streams[:2])])
        for graph, s in zip(graphs, streams[2:]):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for pair in got + [outs]:
        for a, b in zip(pair, want if pair is not outs else want[2:]):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
