"""Calls of a session, a cache and a rotary chained on a stream that is not the default one, without synchronising."""
import pytest
import torch

from paper_2502_03805_b200 import ChunkedPrefillCompressor, CompressionSession, PagedCache, Rotary, rope_frequencies

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator().manual_seed(seed)


def test_the_documented_chain_on_a_side_stream():
    """compact_into between new_lengths and the calls of a decode step, with the default stream held up before the
    compression and the side stream before the lengths: the same bits as on the default stream alone."""
    g = gen(1)
    Hq, Hkv, dh, dm, n, w = 4, 2, 64, 64, 900, 8
    args = [torch.randn(*s, generator=g).bfloat16().cuda() for s in ((1, Hq, w, dh), (1, Hkv, n, dh), (1, Hkv, n, dh), (1, Hq, dh, dm))]
    q, k, v = (torch.randn(1, H, 1, dh, generator=g).bfloat16().cuda() for H in (Hq, Hkv, Hkv))
    pos = torch.full((1, 1), n, dtype=torch.int32, device="cuda")
    rotary = Rotary(dh=dh, frequencies=rope_frequencies(dh), device="cuda:0")

    def chain(wait):
        s = CompressionSession(nb=1, Hq=Hq, Hkv=Hkv, dh=dh, dm=dm, n=n, w=w, pool_k=3, dtype="bf16", budget_mode="adaptive",
                               budget=500)
        cache = PagedCache.allocate(nseq=1, Hq=Hq, Hkv=Hkv, dh=dh, dtype="bf16", rows=n + 8, format="e4m3", page_size=16)
        start = torch.full((1, Hkv), 333, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.default_stream()):
            wait()
        s.compress(*args)
        wait()
        start.zero_()
        lens = s.compact_into(cache, args[1], args[2], start)
        qr, kr = rotary.rotate(q, k, pos)
        lens = cache.store(kr, v, lens, lens)
        return cache.attend(qr[:, :, 0], lens) + (lens,)

    want = [x.cpu() for x in chain(lambda: None)]
    with torch.cuda.stream(torch.cuda.Stream()):
        got = [x.cpu() for x in chain(lambda: torch.cuda._sleep(20_000_000))]     # about 10 ms
    assert int(want[2].sum()) == 500 + Hkv
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("mode", ["uniform", "adaptive"])
def test_a_chunked_prefill_into_a_cache_on_a_side_stream(mode):
    """to_cache with a side stream current, the default stream still busy with what the rows come from."""
    g = gen(2)
    Hq, Hkv, dh, dm, w, n = 4, 2, 64, 64, 8, 90
    ch = ChunkedPrefillCompressor(Hq=Hq, Hkv=Hkv, dh=dh, dm=dm, w=w, pool_k=3, dtype="bf16", budget_mode=mode)
    ch.step(*(torch.randn(*s, generator=g).bfloat16().cuda() for s in ((Hq, w, dh), (Hkv, n, dh), (Hkv, n, dh), (Hq, dh, dm))),
            40 if mode == "uniform" else 80)
    cache = PagedCache.allocate(nseq=1, Hq=Hq, Hkv=Hkv, dh=dh, dtype="bf16", rows=100)
    rows = [ch.K, ch.V] if mode == "uniform" else ch.K + ch.V
    kept = [x.clone() for x in rows]
    for x in rows:
        x.zero_()
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    for x, y in zip(rows, kept):                     # on the default stream, behind the wait
        x.copy_(y)
    with torch.cuda.stream(torch.cuda.Stream()):
        lens = ch.to_cache(cache)
        K, V = (x.cpu() for x in cache.load(lens, 80))
    for h in range(Hkv):
        m = int(lens[0, h])
        assert m == ch.K[h].shape[0]
        assert torch.equal(K[0, h, :m], ch.K[h].cpu()) and torch.equal(V[0, h, :m], ch.V[h].cpu())


def test_a_compression_into_a_cache_captured_as_a_graph():
    """With the captured stream given; each replay selects and stores again."""
    g = gen(5)
    Hq, Hkv, dh, dm, n, w = 4, 2, 64, 64, 300, 8
    Qw, K, V, WO = (torch.randn(*s, generator=g).bfloat16().cuda() for s in ((1, Hq, w, dh), (1, Hkv, n, dh), (1, Hkv, n, dh), (1, Hq, dh, dm)))
    s = CompressionSession(nb=1, Hq=Hq, Hkv=Hkv, dh=dh, dm=dm, n=n, w=w, pool_k=3, dtype="bf16", budget_mode="uniform", budget=60)
    cache = PagedCache.allocate(nseq=1, Hq=Hq, Hkv=Hkv, dh=dh, dtype="bf16", rows=n)
    start, lens = cache.new_lengths(), cache.new_lengths()
    s.compress(Qw, K, V, WO)
    s.compact_into(cache, K, V, start, lens)
    want = [x.clone() for x in cache.load(lens, 60)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        with pytest.raises(ValueError):
            s.compact_into(cache, K, V, start, lens)
        s.compact_into(cache, K, V, start, lens, stream=torch.cuda.current_stream())
    for _ in range(2):
        cache.k_pages.zero_()
        cache.v_pages.zero_()
        lens.zero_()
        graph.replay()
        assert lens.cpu().tolist() == [[60, 60]]
        for a, b in zip(cache.load(lens, 60), want):
            assert torch.equal(a, b)
