"""Appending new tokens with their rotation against rope and store one behind the other (the same bits), and against 64 bits."""
import pytest
import torch

import cache_ref as R
import four_bit as F
from canary_util import Guarded
from paper_2502_03805_b200 import PagedCache, Rotary
from paper_2502_03805_b200 import binding as B
from paper_2502_03805_b200 import rope_frequencies
from test_cache_gpu import Cache, check_rope, gen, same

pytestmark = pytest.mark.gpu
FORMATS = ["plain", "e4m3", "int8", "e2m1"]


def make(fmt, **kw):
    return F.FourBit(**kw) if fmt == "e2m1" else Cache(fmt=fmt, **kw)


def projected(nseq, T, Hq, Hkv, dh, dtype, seed=1):
    """q, k, v as parts of one projection's output, guarded."""
    both = Guarded((nseq, T, Hq + 2 * Hkv, dh), R.DT[dtype])
    both.t.copy_(torch.randn(both.t.shape, generator=gen(seed)).to(R.DT[dtype]))
    q, k, v = (x.transpose(1, 2) for x in both.t.split([Hq, Hkv, Hkv], dim=2))
    return both, q, k, v


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dh,rot,nseq,T,Hq,Hkv,page", [
    (128, 128, 1, 1, 32, 8, 64), (64, 32, 61, 1, 8, 2, 16), (64, 64, 2, 37, 3, 1, 32), (128, 48, 3, 5, 5, 5, 16),
    (128, 16, 1, 130, 2, 2, 256), (64, 20, 2, 9, 6, 3, 16), (128, 6, 1, 33, 4, 4, 128), (128, 112, 2, 3, 1, 1, 16)])
def test_the_same_bits_as_rope_then_store(dtype, fmt, layout, dh, rot, nseq, T, Hq, Hkv, page):
    kw = dict(nseq=nseq, Hq=Hq, Hkv=Hkv, dh=dh, dtype=dtype, page=page, cols=-(-(T + 40) // page))
    one, two = make(fmt, **kw), make(fmt, **kw)
    both, q, k, v = projected(nseq, T, Hq, Hkv, dh, dtype)
    given = both.t.clone()
    pos = torch.randint(-9, 140000, (nseq, T), generator=gen(2), dtype=torch.int32).cuda()
    start = torch.randint(0, 41, (nseq, Hkv), generator=gen(3), dtype=torch.int32).cuda()
    rotary = Rotary(dh=dh, frequencies=rope_frequencies(rot, 500000.0), layout=layout, factor=1.25, device="cuda:0")
    q_out = Guarded((nseq, Hq, T, dh), R.DT[dtype])
    before = B.criticalkv_launch_count(one.c.handle)
    got, lens = one.c.append(q, k, v, pos, rotary, start, q_out=q_out.t)
    assert B.criticalkv_launch_count(one.c.handle) == before + 1
    want_q, want_k = rotary.rotate(q, k, pos)
    want_lens = two.c.store(want_k, v.contiguous(), start)
    assert got is q_out.t and torch.equal(got, want_q) and torch.equal(lens, want_lens)
    assert same(one.bits(), two.bits())
    assert torch.equal(both.t, given) and both.intact() and q_out.intact() and one.intact()
    check_rope(got, q.cpu(), pos.cpu(), rotary.freq.cpu(), layout, 1.25, dtype)
    one.c.append(q, k, v, pos, rotary, start, q_out=q)                        # queries turned where they are
    assert torch.equal(q, want_q) and torch.equal(both.t[:, :, Hq:], given[:, :, Hq:])
    assert same(one.bits(), two.bits()) and both.intact() and one.c.device_status() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout,rot", [("half", 128), ("interleaved", 128), ("half", 36), ("interleaved", 36), ("half", 40),
                                        ("interleaved", 40)])
def test_the_same_bits_on_many_rows(dtype, layout, rot):
    """Sums that are rounded another way differ in a few of ten thousand bf16 results."""
    nseq, Hq, Hkv, T, dh = 1, 16, 4, 4096, 128
    cache = Cache(nseq=nseq, Hq=Hq, Hkv=Hkv, dh=dh, dtype=dtype, fmt="plain", page=64, cols=64)
    q, k, v = (torch.randn(nseq, h, T, dh, generator=gen(h)).to(R.DT[dtype]).cuda() for h in (Hq, Hkv, Hkv))
    pos = torch.arange(T, dtype=torch.int32, device="cuda")[None]
    rotary = Rotary(dh=dh, frequencies=rope_frequencies(rot, 500000.0), layout=layout, device="cuda:0")
    got, lens = cache.c.append(q, k, v, pos, rotary, cache.c.new_lengths())
    want_q, want_k = rotary.rotate(q, k, pos)
    assert torch.equal(got, want_q)
    K, V = cache.c.load(lens, T)
    assert torch.equal(K, want_k) and torch.equal(V, v)


@pytest.mark.parametrize("T", [1, 40, 500])      # the lengths in the same launch, and in a second one
def test_counts_and_lengths_in_place(T):
    nseq, Hq, Hkv, dh = 4, 4, 2, 128
    cache = make("e2m1", nseq=nseq, Hq=Hq, Hkv=Hkv, dh=dh, dtype="bf16", page=32, cols=-(-(T + 9) // 32))
    both, q, k, v = projected(nseq, T, Hq, Hkv, dh, "bf16")
    counts = torch.tensor([T, 0, (T + 1) // 2, 1], dtype=torch.int32)
    lens = torch.tensor([[5, 0], [2, 9], [0, 1], [7, 7]], dtype=torch.int32)
    dev, pos = lens.cuda(), torch.arange(T, dtype=torch.int32, device="cuda").repeat(nseq, 1)
    rotary = Rotary(dh=dh, frequencies=rope_frequencies(dh), device="cuda:0")
    before, q_out = cache.bits(), torch.full((nseq, Hq, T, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    _, out = cache.c.append(q, k, v, pos, rotary, dev, dev, q_out=q_out, counts=counts.cuda())
    assert out is dev and torch.equal(dev.cpu(), lens + counts[:, None])
    want_q, want_k = (x.cpu() for x in rotary.rotate(q, k, pos))
    want = F.expect_store(cache, before, want_k, v.cpu(), lambda s, h: range(int(counts[s])), lens)
    assert same(cache.bits(), want) and cache.intact()
    for s in range(nseq):
        n = int(counts[s])
        assert torch.equal(q_out[s, :, :n].cpu(), want_q[s, :, :n]) and bool((q_out[s, :, n:] == 7.0).all())


@pytest.mark.parametrize("fmt", FORMATS)
def test_places_outside_the_table_or_the_pool_are_skipped_and_reported(fmt):
    nseq, T, H, dh = 1, 20, 4, 64
    cache = make(fmt, nseq=nseq, Hq=H, Hkv=H, dh=dh, dtype="bf16", page=16, cols=3, flags=B.CKV_FLAG_DEBUG_CHECKS)
    other = make(fmt, nseq=nseq, Hq=H, Hkv=H, dh=dh, dtype="bf16", page=16, cols=3)
    cache.table_dev[0, 2, 1], cache.table_dev[0, 1, 0] = -1, cache.k.shape[0]
    other.table_dev.copy_(cache.table_dev)
    both, q, k, v = projected(nseq, T, H, H, dh, "bf16")
    start = torch.tensor([[40, 0, -3, 2 ** 31 - 5]], dtype=torch.int32, device="cuda")
    pos = torch.zeros(1, T, dtype=torch.int32, device="cuda")
    rotary = Rotary(dh=dh, frequencies=rope_frequencies(dh), device="cuda:0")
    q_out, lens = cache.c.append(q, k, v, pos, rotary, start)
    assert cache.c.device_status() == B.CKV_EBOUNDS and cache.intact()
    assert torch.equal(q_out, q) and torch.equal(lens, other.c.store(k.contiguous(), v.contiguous(), start))   # position 0
    assert same(cache.bits(), other.bits())
    assert cache.c.append(q, k, v, pos, rotary, start * 0, counts=torch.tensor([21], dtype=torch.int32, device="cuda"))
    assert cache.c.device_status() == B.CKV_EBOUNDS


def test_special_rows_and_no_tokens():
    """Infinities, NaN and zeros among the new rows, and a call without tokens."""
    nseq, T, dh = 1, 6, 64
    rotary = Rotary(dh=dh, frequencies=rope_frequencies(32), device="cuda:0")
    for fmt in FORMATS:
        one, two = (make(fmt, nseq=1, Hq=1, Hkv=1, dh=dh, dtype="f32", page=16, cols=1) for _ in range(2))
        x = torch.randn(1, 1, T, dh, generator=gen(4))
        x[0, 0, 0], x[0, 0, 1, 3], x[0, 0, 2, 60], x[0, 0, 3, 17] = 0.0, float("inf"), float("nan"), 3e38
        x, pos = x.cuda(), torch.arange(T, dtype=torch.int32, device="cuda")[None]
        start = one.c.new_lengths()
        q, lens = one.c.append(x, x, x, pos, rotary, start)
        want_q, want_k = rotary.rotate(x, x, pos)
        two.c.store(want_k, x, start)
        assert torch.equal(torch.nan_to_num(q), torch.nan_to_num(want_q)) and same(one.bits(), two.bits()) and int(lens) == T
        none = x[:, :, :0]
        q, lens = one.c.append(none, none, none, pos[:, :0].contiguous(), rotary, lens, lens)
        assert q.shape == none.shape and int(lens) == T and same(one.bits(), two.bits())


def test_refusals():
    cache = PagedCache.allocate(nseq=2, Hq=4, Hkv=2, dh=64, dtype="bf16", rows=50)
    rotary = Rotary(dh=64, frequencies=rope_frequencies(64), device="cuda:0")
    q, k, v = (torch.zeros(2, h, 3, 64, dtype=torch.bfloat16, device="cuda") for h in (4, 2, 2))
    pos, start = torch.zeros(2, 3, dtype=torch.int32, device="cuda"), cache.new_lengths()
    ok = dict(q=q, k=k, v=v, positions=pos, rotary=rotary, start=start)
    cache.append(**ok)
    for bad in (dict(q=q.float()), dict(q=q.cpu(), q_out=q), dict(k=k[:, :1]), dict(v=v[:, :, :2]), dict(v=v.half()), dict(q=q[0], q_out=q),
                dict(positions=pos.long()), dict(positions=pos[:, :2]), dict(start=start.long()), dict(start=start[:1]),
                dict(lens_out=start[0]), dict(q_out=q[:, :2]), dict(q_out=q.float()), dict(counts=start),
                dict(k=k[:, :1].expand(2, 2, 3, 64)), dict(positions=pos.t().contiguous().t()),
                dict(rotary=Rotary(dh=128, frequencies=rope_frequencies(128), device="cuda:0")), dict(positions=pos.cpu())):
        with pytest.raises(ValueError):
            cache.append(**{**ok, **bad})
    with pytest.raises(B.CriticalKVError):                        # more turned elements than the row has
        cache.append(**{**ok, "rotary": Rotary(dh=64, frequencies=rope_frequencies(128), device="cuda:0")})
    with pytest.raises(B.CriticalKVError):                        # the lengths written over the positions
        cache.append(**{**ok, "lens_out": pos.view(-1)[1:5].view(2, 2)})
