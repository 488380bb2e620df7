"""Pages in 4 bits a value: store and load bit for bit, decode attention against 64 bits with the bounds of the kernel that ran."""
import math

import pytest
import torch

import cache_ref as R
import decode_bounds as D
import four_bit as F
from canary_util import Guarded
from paper_2502_03805_b200 import CompressionSession, PagedCache
from paper_2502_03805_b200 import binding as B
from test_cache_gpu import LENS, gen, same

pytestmark = pytest.mark.gpu


# ---- rows in and out -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh,page,nseq,Hkv,n,at", [(64, 16, 2, 3, 1, 5), (128, 64, 1, 2, 70, 0), (64, 256, 3, 1, 130, 100),
                                                   (128, 32, 2, 2, 700, 31)])
def test_store_writes_exactly_the_rows_and_load_reads_them(dtype, dh, page, nseq, Hkv, n, at):
    g = gen(n)
    cache = F.FourBit(nseq=nseq, Hq=Hkv, Hkv=Hkv, dh=dh, dtype=dtype, page=page, cols=(n + at + page - 1) // page + 1)
    K, V = ((torch.randn(nseq, Hkv, n, dh, generator=g) * torch.exp(2 * torch.randn(nseq, Hkv, n, dh, generator=g))).to(R.DT[dtype])
            for _ in range(2))
    start = torch.randint(0, at + 1, (nseq, Hkv), generator=g, dtype=torch.int32)
    before = cache.bits()
    lens = cache.c.store(K.cuda(), V.cuda(), start.cuda())
    assert same(cache.bits(), F.expect_store(cache, before, K, V, lambda s, h: range(n), start))
    assert torch.equal(lens.cpu(), start + n) and cache.intact()
    out = [Guarded((nseq, Hkv, n, dh), R.DT[dtype]) for _ in range(2)]
    cache.c.load(lens, K_out=out[0].t, V_out=out[1].t, align_right=True)
    for x, got in zip((K, V), out):
        want = F.values(*F.quantise(x)).float().to(R.DT[dtype])          # code * group scale is exact, one rounding a step
        assert torch.equal(got.t.cpu(), want) and got.intact()


def test_store_of_selected_rows_strided_source_interleaved_pool():
    g = gen(9)
    nseq, Hkv, n, dh = 2, 3, 301, 128
    cache = F.FourBit(nseq=nseq, Hq=Hkv, Hkv=Hkv, dh=dh, dtype="bf16", page=32, cols=8, interleave=True)
    src = torch.randn(nseq, n, 2, Hkv, dh, generator=g).bfloat16()
    dev = src.cuda()
    K, V = src[:, :, 0].transpose(1, 2), src[:, :, 1].transpose(1, 2)
    counts = torch.tensor([[100, 0, 37], [1, 150, 20]])
    chosen = [[torch.randperm(n, generator=g)[:c].sort().values for c in row] for row in counts.tolist()]
    idx = torch.full((nseq, 171 + 4), -1, dtype=torch.int32)
    for s in range(nseq):
        flat = torch.cat(chosen[s])
        idx[s, :len(flat)] = flat.to(torch.int32)
    offsets = torch.nn.functional.pad(counts.cumsum(1), (1, 0)).to(torch.int32)
    start = torch.tensor([[3, 7, 0], [40, 2, 11]], dtype=torch.int32)
    before = cache.bits()
    lens = cache.c.store(dev[:, :, 0].transpose(1, 2), dev[:, :, 1].transpose(1, 2), start.cuda(), idx=idx.cuda(),
                         offsets=offsets.cuda())
    assert same(cache.bits(), F.expect_store(cache, before, K, V, lambda s, h: chosen[s][h], start))
    assert torch.equal(lens.cpu(), (start + counts).to(torch.int32)) and cache.intact()
    q = torch.randn(nseq, Hkv, dh, generator=g).bfloat16()
    lens0 = torch.minimum(lens.cpu(), lens.cpu() - start)                    # the rows in front of `start` are garbage
    full = F.FourBit(nseq=nseq, Hq=Hkv, Hkv=Hkv, dh=dh, dtype="bf16", page=32, cols=8, interleave=True)
    full.c.store(dev[:, :, 0].transpose(1, 2), dev[:, :, 1].transpose(1, 2), full.c.new_lengths(), idx=idx.cuda(),
                 offsets=offsets.cuda())
    check(full, q, lens0.to(torch.int32))


def test_store_of_special_rows():
    """Zeros, the smallest and largest magnitudes, infinities and NaN, ties between codes; what they stand for is read back."""
    for dtype in ("f32", "bf16"):
        top = float(torch.finfo(R.DT[dtype]).max)
        tiny = float(torch.finfo(R.DT[dtype]).smallest_normal)
        rows = torch.randn(11, 64, generator=gen(4))
        rows[0] = 0.0
        rows[1] *= tiny
        rows[2] = top
        rows[3, 5] = math.inf
        rows[4, 6] = -math.inf
        rows[5, 7] = math.nan
        rows[6] = tiny / 8                                                   # subnormal
        rows[7, 1:] = 0.0
        rows[8] = torch.linspace(-1, 1, 64)
        rows[9] = torch.arange(64) % 29 * 0.25 * torch.where(torch.arange(64) % 2 == 0, 1.0, -1.0)   # halfway between codes
        rows[9, ::16] = 6.0
        rows[10, 16:] *= 2.0 ** -18                                          # groups whose scale vanishes beside the row's
        rows = rows.to(R.DT[dtype])
        cache = F.FourBit(nseq=1, Hq=1, Hkv=1, dh=64, dtype=dtype, page=16, cols=1)
        x = rows.cuda()[None, None]
        lens = cache.c.store(x, x, torch.zeros(1, 1, dtype=torch.int32, device="cuda"))
        page = int(cache.table[0, 0, 0])
        code, group, scale = F.quantise(rows)
        assert torch.equal(torch.nan_to_num(cache.ks[page, :11].cpu(), nan=-1.0), torch.nan_to_num(scale, nan=-1.0))
        assert torch.equal(cache.k[page, :11].cpu(), code)
        assert torch.equal(cache.kg.view(torch.uint8)[page, :11].cpu(), group.view(torch.uint8))
        finite = torch.isfinite(rows.float()).all(-1)
        back = cache.c.load(lens, 11)[1][0, 0].cpu()
        assert bool(torch.isnan(back[~finite]).all()) and bool(torch.isfinite(back[finite]).all())
        assert torch.equal(back[finite], F.values(code, group, scale)[finite].float().to(R.DT[dtype]))


def test_store_outside_the_table_or_the_pool_is_skipped_and_reported():
    g = gen(6)
    cache = F.FourBit(nseq=1, Hq=4, Hkv=4, dh=64, dtype="bf16", page=16, cols=3, flags=B.CKV_FLAG_DEBUG_CHECKS)
    n = 20
    K, V = (torch.randn(1, 4, n, 64, generator=g).bfloat16() for _ in range(2))
    start = torch.tensor([[40, 0, -3, 2 ** 31 - 5]], dtype=torch.int32)
    before = cache.bits()
    lens = cache.c.store(K.cuda(), V.cuda(), start.cuda())
    assert cache.c.device_status() == B.CKV_EBOUNDS
    assert same(cache.bits(), F.expect_store(cache, before, K, V, lambda s, h: range(n), start)) and cache.intact()
    assert lens.cpu().tolist() == [[48, 20, 17, 48]]
    bad = cache.table_dev.clone()
    bad[0, 1, 0], bad[0, 2, 1] = -1, cache.k.shape[0]
    cache.table_dev.copy_(bad)
    cache.c.store(K.cuda(), V.cuda(), torch.zeros_like(start).cuda())
    assert cache.c.device_status() == B.CKV_EBOUNDS and cache.intact()


# ---- attention -------------------------------------------------------------------------------------------------------
def check(cache, q, lens, c=None, kernel=None, scale=None, given=None):
    c = cache.c if c is None else c
    got = c.attend(q.cuda(), (lens if given is None else given).cuda())
    kernel = kernel or "tensor"
    assert B.criticalkv_last_path(c.handle) & 384 == (128 if kernel == "tensor" else 256)
    want = F.attention(q, cache, lens, 1.0 / math.sqrt(cache.dh) if scale is None else scale, kernel)
    D.check(got, want, lens, q.shape[1] // cache.Hkv)
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh,G,Hkv,nseq,page,lens", [
    (128, 4, 8, 1, 64, "ragged"), (64, 1, 2, 5, 16, "short"), (128, 8, 2, 8, 32, "edges"), (64, 5, 3, 6, 128, "edges"),
    (128, 1, 1, 1, 16, "one"), (64, 12, 2, 3, 64, "ragged"), (128, 16, 1, 2, 256, "ragged"), (128, 40, 1, 3, 16, "ragged"),
    (64, 32, 2, 2, 32, "short"), (128, 5, 8, 40, 16, "ragged")])
@pytest.mark.parametrize("size", [0.1, 1.5])
def test_shapes(dtype, dh, G, Hkv, nseq, page, lens, size):
    lens = LENS[lens](nseq, Hkv)
    cols = max(1, -(-int(lens.max()) // page))
    cache = F.FourBit(nseq=nseq, Hq=G * Hkv, Hkv=Hkv, dh=dh, dtype=dtype, page=page, cols=cols, seed=dh + G).fill(lens, G)
    q = (size * torch.randn(nseq, G * Hkv, dh, generator=gen(G + 1))).to(R.DT[dtype])
    got = check(cache, q, lens)
    again = cache.c.attend(q.cuda(), lens.cuda())
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    check(cache, q, lens, cache.other(flags=B.CKV_FLAG_FORCE_SIMT), "cuda")
    assert cache.intact()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("G,nseq,Hkv,lens", [(3, 1, 1, [[30011]]), (4, 2, 2, [[20011, 3], [0, 1]]),
                                             (2, 3, 3, [[7000, 1, 64], [0, 9000, 129], [12000, 65, 63]])])
def test_long_heads(dtype, dh, G, nseq, Hkv, lens):
    lens = torch.tensor(lens, dtype=torch.int32)
    cache = F.FourBit(nseq=nseq, Hq=G * Hkv, Hkv=Hkv, dh=dh, dtype=dtype, page=128, cols=235).fill(lens, 3)
    check(cache, torch.randn(nseq, G * Hkv, dh, generator=gen(8)).to(R.DT[dtype]), lens)


@pytest.mark.parametrize("dh,G,page,lens", [(128, 4, 16, "short"), (64, 8, 64, "edges"), (128, 16, 32, "edges")])
def test_many_short_heads_and_a_long_one(dh, G, page, lens):
    nseq, Hkv = 60, 8
    lens = LENS[lens](nseq, Hkv)
    lens[31, 3] = 3001
    cache = F.FourBit(nseq=nseq, Hq=G * Hkv, Hkv=Hkv, dh=dh, dtype="bf16", page=page, cols=-(-3001 // page)).fill(lens, G)
    check(cache, (1.5 * torch.randn(nseq, G * Hkv, dh, generator=gen(G + 1))).bfloat16(), lens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,G,Hkv", [(128, 4, 2), (64, 16, 1), (64, 8, 25)])
@pytest.mark.parametrize("rows", [16, 48, 384, 1300])
def test_clusters_and_none(dtype, dh, G, Hkv, rows):
    cache = F.FourBit(nseq=1, Hq=G * Hkv, Hkv=Hkv, dh=dh, dtype=dtype, page=16, cols=(rows + 15) // 16)
    full = torch.full((1, Hkv), rows, dtype=torch.int32)
    cache.fill(full, 2)
    apart = cache.other(flags=B.CKV_FLAG_SELECT_NO_CLUSTER)
    q = torch.randn(1, G * Hkv, dh, generator=gen(3)).to(R.DT[dtype])
    for lens in (full, torch.zeros_like(full), (full - torch.arange(Hkv) * 7).clamp(min=0).to(torch.int32)):
        check(cache, q, lens)
        check(cache, q, lens, apart)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_of_very_different_size(dtype):
    lens = torch.tensor([[200, 97]], dtype=torch.int32)
    cache = F.FourBit(nseq=1, Hq=4, Hkv=2, dh=64, dtype=dtype, page=32, cols=7).fill(lens, 3, spread=4.0)
    check(cache, (3 * torch.randn(1, 4, 64, generator=gen(8))).to(R.DT[dtype]), lens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("size", [2.0 ** 40, 2.0 ** -40, 0.0])
def test_large_and_tiny_queries(dtype, dh, size):
    lens = torch.full((1, 1), 40, dtype=torch.int32)
    scale = 1.0 / (8 * size) if size else 1.0
    cache = F.FourBit(nseq=1, Hq=2, Hkv=1, dh=dh, dtype=dtype, page=16, cols=3, scale=scale).fill(lens, 3)
    check(cache, (size * torch.randn(1, 2, dh, generator=gen(8))).to(R.DT[dtype]), lens, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("order", ["rising", "falling", "one late"])
def test_logits_that_keep_growing(dtype, order):
    """References that move: logits that rise by a little, by a lot, and a lone large one behind many small ones; a head
    whose first rows score -infinity and below any reference."""
    n, dh = 900, 64
    lens = torch.full((1, 2), n, dtype=torch.int32)
    cache = F.FourBit(nseq=1, Hq=4, Hkv=2, dh=dh, dtype=dtype, page=32, cols=29, scale=1.0).fill(lens, 3)
    g = gen(4)
    size = {"rising": torch.linspace(-60, 60, n), "falling": torch.linspace(60, -60, n),
            "one late": torch.where(torch.arange(n) == 871, 90.0, 0.01)}[order]
    for h in range(2):
        k = torch.randn(n, dh, generator=g) * 0.02
        k[:, 0] = size / (1 + h)
        v = torch.randn(n, dh, generator=g) * torch.exp(4 * torch.randn(n, 1, generator=g))
        cache.put(0, h, torch.arange(n), (k.to(R.DT[dtype]), v.to(R.DT[dtype])))
    q = 0.1 * torch.randn(1, 4, dh, generator=g)
    q[:, :, 0] = torch.tensor([1.0, -1.0, 0.3, 2.0])
    check(cache, q.to(R.DT[dtype]), lens, scale=1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_absent_pages_wild_lengths_and_empty_heads(dtype):
    lens = torch.tensor([[48, 48, 30]], dtype=torch.int32)
    cache = F.FourBit(nseq=1, Hq=6, Hkv=3, dh=64, dtype=dtype, page=16, cols=3, flags=B.CKV_FLAG_DEBUG_CHECKS).fill(lens, 3)
    q = torch.randn(1, 6, 64, generator=gen(8)).to(R.DT[dtype])
    check(cache, q, torch.tensor([[48, 48, 0]], dtype=torch.int32), given=torch.tensor([[2 ** 31 - 1, 49, -5]], dtype=torch.int32))
    assert cache.c.device_status() == B.CKV_EBOUNDS
    cache.table_dev[0, 0, 2], cache.table_dev[0, 1, 2], cache.table_dev[0, 2] = -1, cache.k.shape[0], -7
    got = cache.c.attend(q.cuda(), lens.cuda())
    want = F.attention(q, cache, torch.tensor([[32, 32, 0]]), 0.125, "tensor")
    assert bool(((got[0].cpu().double() - want[0]).abs() <= want[2])[0, :4].all())
    assert bool(torch.isnan(got[0][0, 4:]).all())                             # rows, but none in an existing page
    assert cache.c.device_status() == B.CKV_EBOUNDS and cache.intact()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinities_and_nan_spoil_only_the_heads_that_read_them(dtype):
    lens = torch.tensor([[70, 70, 70, 70]], dtype=torch.int32)
    cache = F.FourBit(nseq=1, Hq=4, Hkv=4, dh=64, dtype=dtype, page=16, cols=5).fill(lens, 3)
    rows = torch.randn(4, 64, generator=gen(5)).to(R.DT[dtype])
    bad = rows.clone()
    bad[0, 3], bad[1, 40] = math.nan, -math.inf
    cache.put(0, 1, torch.arange(30, 34), (rows, bad))
    cache.put(0, 2, torch.arange(66, 70), (bad, rows))
    q = torch.randn(1, 4, 64, generator=gen(8)).to(R.DT[dtype])
    out, lse = (x.cpu() for x in cache.c.attend(q.cuda(), lens.cuda()))
    assert bool(torch.isnan(out[0, 1]).all()) and bool(torch.isfinite(lse[0, 1]))
    assert bool(torch.isnan(out[0, 2]).all()) and bool(torch.isnan(lse[0, 2]))
    for h in (0, 3):
        assert bool(torch.isfinite(out[0, h]).all()) and bool(torch.isfinite(lse[0, h]))


def test_strided_queries_own_page_stride_and_shared_pages():
    lens = torch.tensor([[50, 20], [50, 33]], dtype=torch.int32)
    cache = F.FourBit(nseq=2, Hq=8, Hkv=2, dh=64, dtype="bf16", page=16, cols=4, scale=0.31, interleave=True).fill(lens, 3)
    cache.table[1, 0] = cache.table[0, 0]
    cache.table_dev.copy_(cache.table)
    both = torch.randn(2, 12, 64, generator=gen(8)).bfloat16()
    got = cache.c.attend(both.cuda()[:, 2:10], lens.cuda())
    want = F.attention(both[:, 2:10], cache, lens, 0.31, "tensor")
    D.check(got, want, lens, 4)


def test_a_compressed_prompt_goes_into_four_bits():
    """The compression step's selection, written to 4-bit pages and attended to."""
    g = gen(12)
    n, dh, dm = 512, 64, 256
    s = CompressionSession(nb=2, Hq=4, Hkv=2, dh=dh, dm=dm, n=n, w=16, pool_k=5, dtype="bf16", budget_mode="adaptive", budget=300)
    Qw, K, V, WO = (torch.randn(shape, generator=g).bfloat16() for shape in
                    ((2, 4, 16, dh), (2, 2, n, dh), (2, 2, n, dh), (2, 4, dh, dm)))
    s.compress(Qw.cuda(), K.cuda(), V.cuda(), WO.cuda())
    cache = F.FourBit(nseq=2, Hq=4, Hkv=2, dh=dh, dtype="bf16", page=32, cols=16)
    before = cache.bits()
    lens = s.compact_into(cache.c, K.cuda(), V.cuda(), cache.c.new_lengths())
    off = s.offsets.cpu()
    rows = lambda b, h: s.idx[b, off[b, h]:off[b, h + 1]].cpu().tolist()  # noqa: E731
    assert same(cache.bits(), F.expect_store(cache, before, K, V, rows, torch.zeros(2, 2, dtype=torch.int32)))
    check(cache, torch.randn(2, 4, dh, generator=g).bfloat16(), lens.cpu())


def test_allocated_pool_and_refusals():
    cache = PagedCache.allocate(nseq=1, Hq=2, Hkv=1, dh=128, dtype="bf16", rows=100, format="e2m1")
    assert cache.k_pages.shape == (2, 64, 64) and cache.k_group_scale.shape == (2, 64, 8)
    K = torch.randn(1, 1, 100, 128, generator=gen(1)).bfloat16()
    lens = cache.store(K.cuda(), K.cuda(), cache.new_lengths())
    back, _ = cache.load(lens, 100)
    assert torch.equal(back.cpu(), F.values(*F.quantise(K)).float().bfloat16())
    ok = dict(Hq=2, dtype="bf16", format="e2m1", k_pages=cache.k_pages, v_pages=cache.v_pages, k_scale=cache.k_scale,
              v_scale=cache.v_scale, k_group_scale=cache.k_group_scale, v_group_scale=cache.v_group_scale,
              page_table=cache.page_table)
    PagedCache(**ok)
    for bad in (dict(k_group_scale=None), dict(v_scale=None), dict(k_group_scale=cache.k_group_scale[:1]),
                dict(v_group_scale=cache.v_group_scale.view(torch.uint8)), dict(k_pages=cache.k_pages.view(torch.int8)),
                dict(k_pages=cache.k_pages[..., :32], v_pages=cache.v_pages[..., :32]), dict(format="e4m3"),
                dict(format="plain"), dict(k_group_scale=cache.k_group_scale.transpose(0, 1)),
                dict(k_pages=cache.k_pages[:, ::2], v_pages=cache.v_pages[:, ::2])):
        with pytest.raises(ValueError):
            PagedCache(**{**ok, **bad})
    with pytest.raises(B.CriticalKVError):
        B.criticalkv_decode_workspace_bytes(B.make_cache(nseq=1, Hq=1, Hkv=1, dh=128, dtype="bf16", format="e2m1", page_size=16,
                                                         num_pages=1, max_pages=1, k_pages=256, v_pages=256, page_table=256,
                                                         k_scale=256, v_scale=256, k_group_scale=256, v_group_scale=264))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("right", [False, True])
@pytest.mark.parametrize("n", [1, 37, 200])
def test_load_into_new_tensors_zeroes_what_has_no_row(dtype, right, n):
    """Rows in front of and behind a head's, and those of pages outside the pool; a caller's tensors keep theirs."""
    lens = torch.tensor([[100, 0, 3], [37, 200, 64]], dtype=torch.int32)
    cache = F.FourBit(nseq=2, Hq=3, Hkv=3, dh=64, dtype=dtype, page=16, cols=13).fill(lens, 3)
    for fmt in ("e2m1", "plain"):
        if fmt == "plain":
            c = PagedCache.allocate(nseq=2, Hq=3, Hkv=3, dh=64, dtype=dtype, rows=200, page_size=16)
            rows = cache.c.load(lens.cuda(), 200)
            c.store(*rows, c.new_lengths())
        else:
            c = cache.c
        c.page_table[1, 2, 3] = -1                     # rows 48 to 63
        junk = torch.full((1 << 22,), 7.0, device="cuda")
        del junk                                       # what new tensors are made of
        given = [torch.full((2, 3, n, 64), 5.0, dtype=R.DT[dtype], device="cuda") for _ in range(2)]
        c.load(lens.cuda(), K_out=given[0], V_out=given[1], align_right=right)
        for new, old in zip(c.load(lens.cuda(), n, align_right=right), given):
            at = torch.arange(n).expand(2, 3, n) - ((n - lens.clamp(max=n))[..., None] if right else 0)
            row = at + ((lens - lens.clamp(max=n))[..., None] if right else 0)
            there = (at >= 0) & (at < lens.clamp(max=n)[..., None])
            there[1, 2] &= ~((row[1, 2] >= 48) & (row[1, 2] < 64))
            assert bool((new.cpu()[~there] == 0).all()) and bool((old.cpu()[~there] == 5.0).all())
            assert torch.equal(new.cpu()[there], old.cpu()[there])
