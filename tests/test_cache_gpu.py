"""Rotary positions, the paged cache and decode attention on the GPU against the plain forms of cache_ref.py."""
import math

import numpy as np
import pytest
import torch

import cache_ref as R
from canary_util import Guarded
from paper_2502_03805_b200 import ChunkedPrefillCompressor, CompressionSession, PagedCache, Rotary
from paper_2502_03805_b200 import binding as B
from paper_2502_03805_b200 import rope_frequencies

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -23


def gen(seed):
    return torch.Generator().manual_seed(seed)


# ---- rotary positions ----------------------------------------------------------------------------------------------
def rope_tol(x, want, layout, half, dtype, factor):
    """|a| and |b| of a pair times the error of a cosine or sine (the reduced angle is rounded to float32: 2 pi 2^-26;
    sincospi: 2 ulp; factor: half an ulp) and three roundings of the sum, plus the rounding of the result."""
    ia = torch.arange(half) if layout == "half" else 2 * torch.arange(half)
    ib = ia + (half if layout == "half" else 1)
    both = x.double().abs()[..., ia] + x.double().abs()[..., ib]
    tol = want.abs() * R.HALF_STEP[dtype] + 1e-40
    e = both * abs(factor) * (2 * math.pi * 2.0 ** -26 + 4 * EPS)
    tol[..., ia] += e
    tol[..., ib] += e
    return tol


def check_rope(got, x, pos, freq, layout, factor, dtype):
    want = R.rope(x, pos, freq, layout, factor)
    assert got.shape == want.shape
    bad = (got.cpu().double() - want).abs() > rope_tol(x, want, layout, freq.numel(), dtype, factor)
    assert not bool(bad.any())
    rot = 2 * freq.numel()
    assert torch.equal(got.cpu()[..., rot:], x[..., rot:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("nseq,Hq,Hk,T,dh,rot", [
    (1, 32, 8, 1, 128, 128), (3, 5, 1, 17, 64, 64), (2, 8, 2, 33, 128, 64), (1, 2, 2, 100, 64, 6), (7, 4, 4, 1, 64, 20),
    (1, 1, 1, 3, 8, 2), (1, 3, 1, 5, 256, 256), (2, 1, 1, 16, 96, 48), (40, 12, 3, 1, 64, 32),
    (1, 2, 2, 9, 40, 16), (2, 9, 1, 70, 24, 16), (1, 1, 0, 5, 16, 16), (3, 70, 0, 2, 128, 32)])
def test_rope_shapes(dtype, layout, nseq, Hq, Hk, T, dh, rot):
    g = gen(1)
    q, k = (torch.randn(nseq, H, T, dh, generator=g).to(R.DT[dtype]) for H in (Hq, Hk))
    pos = torch.randint(0, 140000, (nseq, T), generator=g, dtype=torch.int32)
    freq = rope_frequencies(rot, 500000.0)
    r = Rotary(dh=dh, frequencies=freq, layout=layout, device="cuda:0")
    qo, ko = r.rotate(q.cuda(), k.cuda() if Hk else None, pos.cuda())
    check_rope(qo, q, pos, freq, layout, 1.0, dtype)
    if Hk:
        check_rope(ko, k, pos, freq, layout, 1.0, dtype)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_strides_in_place_factor_and_guard_zones(layout):
    g = gen(2)
    nseq, T, Hq, Hk, dh, rot = 2, 21, 6, 2, 64, 32
    both = torch.randn(nseq, T, Hq + 2 * Hk, dh, generator=g).bfloat16()
    pos = torch.randint(-50, 3000, (nseq, T), generator=g, dtype=torch.int32)
    freq = rope_frequencies(rot, 10000.0, "yarn", factor=4.0, original=1024)
    r = Rotary(dh=dh, frequencies=freq, layout=layout, factor=1.25, device="cuda:0")
    buf = Guarded(both.shape, torch.bfloat16)
    buf.t.copy_(both)
    q, k = buf.t[:, :, :Hq].transpose(1, 2), buf.t[:, :, Hq:Hq + Hk].transpose(1, 2)
    out_q, out_k = Guarded((nseq, Hq, T, dh), torch.bfloat16), Guarded((nseq, Hk, T, dh), torch.bfloat16)
    r.rotate(q, k, pos.cuda(), out_q.t, out_k.t)
    check_rope(out_q.t, both[:, :, :Hq].transpose(1, 2), pos, freq, layout, 1.25, "bf16")
    check_rope(out_k.t, both[:, :, Hq:Hq + Hk].transpose(1, 2), pos, freq, layout, 1.25, "bf16")
    assert torch.equal(buf.t.cpu(), both)                       # inputs untouched
    r.rotate(q, k, pos.cuda(), q, k)                            # in place, strided: the same bits
    assert torch.equal(q, out_q.t) and torch.equal(k, out_k.t)
    assert torch.equal(buf.t[:, :, Hq + Hk:].cpu(), both[:, :, Hq + Hk:])
    assert buf.intact() and out_q.intact() and out_k.intact()


def test_rope_without_keys_far_positions_and_back():
    g = gen(3)
    q = torch.randn(1, 4, 8, 128, generator=g)
    top = 2 ** 31 - 1
    pos = torch.tensor([[0, 1, -1, 131072, 10 ** 6, 10 ** 9, top, -top]], dtype=torch.int32)
    freq = rope_frequencies(128, 10000.0)
    r = Rotary(dh=128, frequencies=freq, device="cuda:0")
    out, none = r.rotate(q.cuda(), None, pos.cuda())
    assert none is None
    # the float64 product of position and frequency is itself off by up to 2^-52 of the angle: 2^31 * 2^-52 = 5e-7
    want = R.rope(q, pos, freq, "half")
    assert float((out.cpu().double() - want).abs().max()) < 4e-6 + 1e-6
    back, _ = r.rotate(out, None, -pos.cuda())
    # two turns: twice the error of one, on values of the size of q's (|a| + |b| <= 2 max|q|)
    assert float((back.cpu() - q).abs().max()) < 2 * 2 * float(q.abs().max()) * (2 * math.pi * 2.0 ** -26 + 4 * EPS) + 2e-6


def test_rope_empty_and_refused():
    r = Rotary(dh=64, frequencies=rope_frequencies(64), device="cuda:0")
    q = torch.zeros(2, 3, 0, 64, device="cuda")
    assert r.rotate(q, None, torch.zeros(2, 0, dtype=torch.int32, device="cuda"))[0].shape == q.shape
    q = torch.zeros(2, 3, 4, 64, device="cuda")
    pos = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    for args in ((q.cpu(), None, pos), (q, None, pos.long()), (q, None, pos[:1]), (q.half(), None, pos),
                 (q[..., :32], None, pos), (q, q.bfloat16(), pos), (q[:, :1].expand(2, 3, 4, 64), None, pos),
                 (q, None, pos.cpu())):
        with pytest.raises(ValueError):
            r.rotate(*args)
    with pytest.raises(ValueError):
        Rotary(dh=64, frequencies=rope_frequencies(64).float(), device="cuda:0")
    with pytest.raises(B.CriticalKVError):                        # more rotated elements than the row has
        Rotary(dh=64, frequencies=rope_frequencies(128), device="cuda:0").rotate(q, None, pos)


# ---- a cache for tests -----------------------------------------------------------------------------------------------
class Cache:
    """Pages in guarded buffers, filled with garbage (NaN codes included) wherever no row is stored."""

    def __init__(self, *, nseq, Hq, Hkv, dh, dtype, fmt, page, cols, seed=0, spare=2, interleave=False, flags=0, scale=0.0):
        self.fmt, self.dtype, self.page, self.dh, self.Hkv = fmt, dtype, page, dh, Hkv
        g = gen(seed)
        n = nseq * Hkv * cols + spare
        self.table = torch.randperm(n, generator=g)[:nseq * Hkv * cols].view(nseq, Hkv, cols).to(torch.int32)
        code = R.CODE.get(fmt, R.DT[dtype])
        if interleave:                                            # K and V pages side by side in one pool
            self.pool = Guarded((n, 2, page, dh), code)
            self.k, self.v = self.pool.t[:, 0], self.pool.t[:, 1]
            self.guards = [self.pool]
        else:
            self.guards = [Guarded((n, page, dh), code) for _ in range(2)]
            self.k, self.v = (x.t for x in self.guards)
        raw = torch.uint8 if fmt != "plain" else {2: torch.int16, 4: torch.int32}[code.itemsize]
        self.k.view(raw).fill_(0x7f if fmt != "plain" else -1)    # NaN in every format but int8
        self.v.view(raw).fill_(0x7f if fmt != "plain" else -1)
        self.ks = self.vs = None
        if fmt != "plain":
            s = [Guarded((n, page), torch.float32, fill=math.nan) for _ in range(2)]
            self.guards += s
            self.ks, self.vs = s[0].t, s[1].t
        self.table_dev = self.table.cuda()
        self.c = PagedCache(Hq=Hq, dtype=dtype, format=fmt, k_pages=self.k, v_pages=self.v, k_scale=self.ks,
                            v_scale=self.vs, page_table=self.table_dev, flags=flags, scale=scale)

    def fill(self, lens, seed, spread=1.0):
        """Random rows 0..lens-1 in every head, written on the host side of the test (not by the library)."""
        g = gen(seed)
        k, v = self.k.cpu(), self.v.cpu()
        ks, vs = (x.cpu() if x is not None else None for x in (self.ks, self.vs))
        for s in range(lens.shape[0]):
            for h in range(self.Hkv):
                n = int(lens[s, h])
                if n == 0:
                    continue
                i = torch.arange(n)
                page, slot = self.table[s, h].long()[i // self.page], i % self.page
                for pages, scales in ((k, ks), (v, vs)):
                    x = torch.randn(n, self.dh, generator=g) * torch.exp(spread * torch.randn(n, 1, generator=g))
                    x = x.to(R.DT[self.dtype])
                    if self.fmt == "plain":
                        pages[page, slot] = x
                    else:
                        code, scale = R.quantise(x, self.fmt)
                        pages.view(torch.uint8)[page, slot] = code.view(torch.uint8)
                        scales[page, slot] = scale
        self.k.copy_(k)
        self.v.copy_(v)
        if ks is not None:
            self.ks.copy_(ks)
            self.vs.copy_(vs)
        return self

    def values(self):
        return R.stored(self.k, self.ks, self.fmt), R.stored(self.v, self.vs, self.fmt)

    def intact(self):
        return all(g.intact() for g in self.guards)

    def bits(self):
        return [x.contiguous().view(torch.uint8).cpu() for x in (self.k, self.v, self.ks, self.vs) if x is not None]


FORMATS = ["plain", "e4m3", "int8"]


def expect_store(cache, before, K, V, rows_of, start):
    """The pages as they must look after a store: `before` (bits) with the rows rows_of(s, h) written behind start."""
    want = [b.clone() for b in before]
    cap = cache.table.shape[2] * cache.page
    for s in range(K.shape[0]):
        for h in range(cache.Hkv):
            src = torch.as_tensor(rows_of(s, h), dtype=torch.long)
            to = int(start[s, h]) + torch.arange(len(src))
            keep = (to >= 0) & (to < cap) & (src >= 0) & (src < K.shape[2])
            src, to = src[keep], to[keep]
            page, slot = cache.table[s, h].long()[to // cache.page], to % cache.page
            for j, x in enumerate((K[s, h, src], V[s, h, src])):
                if cache.fmt == "plain":
                    want[j].view(R.DT[cache.dtype]).view(cache.k.shape)[page, slot] = x
                else:
                    code, scale = R.quantise(x, cache.fmt)
                    want[j].view(cache.k.shape)[page, slot] = code.view(torch.uint8)
                    want[2 + j].view(torch.float32).view(cache.ks.shape)[page, slot] = scale
    return want


def same(got, want):
    return all(torch.equal(a.view(-1), b.view(-1)) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh,page,nseq,Hkv,n,at", [(64, 16, 2, 3, 1, 5), (128, 64, 1, 2, 70, 0), (64, 256, 3, 1, 130, 100),
                                                   (128, 32, 2, 2, 700, 31)])
def test_store_writes_exactly_the_rows(dtype, fmt, dh, page, nseq, Hkv, n, at):
    g = gen(n)
    cache = Cache(nseq=nseq, Hq=Hkv, Hkv=Hkv, dh=dh, dtype=dtype, fmt=fmt, page=page, cols=(n + at + page - 1) // page + 1)
    K, V = (torch.randn(nseq, Hkv, n, dh, generator=g).to(R.DT[dtype]) for _ in range(2))
    start = torch.randint(0, at + 1, (nseq, Hkv), generator=g, dtype=torch.int32)
    before = cache.bits()
    lens = cache.c.store(K.cuda(), V.cuda(), start.cuda())
    assert same(cache.bits(), expect_store(cache, before, K, V, lambda s, h: range(n), start))
    assert torch.equal(lens.cpu(), start + n) and cache.intact()


@pytest.mark.parametrize("fmt", FORMATS)
def test_store_of_selected_rows_strided_source_interleaved_pool(fmt):
    g = gen(9)
    nseq, Hkv, n, dh = 2, 3, 301, 128
    cache = Cache(nseq=nseq, Hq=Hkv, Hkv=Hkv, dh=dh, dtype="bf16", fmt=fmt, page=32, cols=8, interleave=True)
    src = torch.randn(nseq, n, 2, Hkv, dh, generator=g).bfloat16()          # token-major, K and V side by side
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
    assert same(cache.bits(), expect_store(cache, before, K, V, lambda s, h: chosen[s][h], start))
    assert torch.equal(lens.cpu(), (start + counts).to(torch.int32)) and cache.intact()


def test_store_of_the_same_row_several_times():
    g = gen(31)
    cache = Cache(nseq=1, Hq=1, Hkv=1, dh=64, dtype="f32", fmt="e4m3", page=16, cols=2)
    K, V = (torch.randn(1, 1, 4, 64, generator=g) for _ in range(2))
    rows = [2, 2, 0, 2, 3, 0, 0]
    before = cache.bits()
    lens = cache.c.store(K.cuda(), V.cuda(), cache.c.new_lengths(), idx=torch.tensor([rows], dtype=torch.int32, device="cuda"),
                         offsets=torch.tensor([[0, 7]], dtype=torch.int32, device="cuda"))
    assert int(lens) == 7
    assert same(cache.bits(), expect_store(cache, before, K, V, lambda s, h: rows, torch.zeros(1, 1, dtype=torch.int32)))


@pytest.mark.parametrize("n", [1, 5000])      # one CTA a head, and many (a second launch then updates the lengths)
def test_store_updates_its_own_lengths_and_honours_counts(n):
    g = gen(n)
    nseq, Hkv, dh = 3, 2, 64
    cache = Cache(nseq=nseq, Hq=2, Hkv=Hkv, dh=dh, dtype="bf16", fmt="e4m3", page=64, cols=2 * n // 64 + 2)
    K, V = (torch.randn(nseq, Hkv, n, dh, generator=g).bfloat16() for _ in range(2))
    counts = torch.tensor([n, 0, (n + 1) // 2], dtype=torch.int32)
    lens = torch.tensor([[5, 0], [2, 9], [n, 1]], dtype=torch.int32)
    dev, before = lens.cuda(), cache.bits()
    out = cache.c.store(K.cuda(), V.cuda(), dev, dev, counts=counts.cuda())
    assert out is dev and torch.equal(dev.cpu(), lens + counts[:, None])
    assert same(cache.bits(), expect_store(cache, before, K, V, lambda s, h: range(int(counts[s])), lens))
    assert cache.intact()


def test_store_of_special_rows():
    """Zeros, the smallest and largest magnitudes, infinities and NaN; what they stand for is read back."""
    for dtype in ("f32", "bf16"):
        top = float(torch.finfo(R.DT[dtype]).max)
        tiny = float(torch.finfo(R.DT[dtype]).smallest_normal)
        rows = torch.randn(9, 64, generator=gen(4))
        rows[0] = 0.0
        rows[1] *= tiny
        rows[2] = top
        rows[3, 5] = math.inf
        rows[4, 6] = -math.inf
        rows[5, 7] = math.nan
        rows[6] = tiny / 8                                                   # subnormal
        rows[7, 1:] = 0.0
        rows[8] = torch.linspace(-1, 1, 64)
        rows = rows.to(R.DT[dtype])
        for fmt in ("e4m3", "int8"):
            cache = Cache(nseq=1, Hq=1, Hkv=1, dh=64, dtype=dtype, fmt=fmt, page=16, cols=1)
            start = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
            x = rows.cuda()[None, None]
            lens = cache.c.store(x, x, start)
            page = int(cache.table[0, 0, 0])
            code, scale = R.quantise(rows, fmt)
            assert torch.equal(torch.nan_to_num(cache.ks[page, :9].cpu(), nan=-1.0), torch.nan_to_num(scale, nan=-1.0))
            finite = torch.isfinite(rows.float()).all(-1)
            assert torch.equal(cache.k[page, :9].cpu().view(torch.uint8)[finite], code.view(torch.uint8)[finite])
            back, _ = cache.c.load(lens, 9)
            back = back[0, 0].cpu()
            assert bool(torch.isnan(back[~finite]).all()) and bool(torch.isfinite(back[finite]).all())
            want = (code.float() * scale[:, None]).to(R.DT[dtype])
            assert torch.equal(back[finite], want[finite])


def test_store_outside_the_table_or_the_pool_is_skipped_and_reported():
    g = gen(6)
    cache = Cache(nseq=1, Hq=4, Hkv=4, dh=64, dtype="bf16", fmt="int8", page=16, cols=3, flags=B.CKV_FLAG_DEBUG_CHECKS)
    good = cache.table_dev.clone()
    n = 20
    K, V = (torch.randn(1, 4, n, 64, generator=g).bfloat16() for _ in range(2))
    start = torch.tensor([[40, 0, -3, 2 ** 31 - 5]], dtype=torch.int32)        # beyond, fits, before row 0, far beyond
    before = cache.bits()
    lens = cache.c.store(K.cuda(), V.cuda(), start.cuda())
    assert cache.c.device_status() == B.CKV_EBOUNDS
    assert same(cache.bits(), expect_store(cache, before, K, V, lambda s, h: range(n), start)) and cache.intact()
    assert lens.cpu().tolist() == [[48, 20, 17, 48]]
    # page ids outside the pool
    bad = good.clone()
    bad[0, 1, 0], bad[0, 2, 1] = -1, cache.k.shape[0]
    cache.table_dev.copy_(bad)
    before = cache.bits()
    cache.c.store(K.cuda(), V.cuda(), torch.zeros_like(start).cuda())
    assert cache.c.device_status() == B.CKV_EBOUNDS and cache.intact()
    after, table = cache.bits(), cache.table.clone()
    want = expect_store(cache, before, K, V, lambda s, h: range(n), torch.zeros_like(start))
    for h, col in ((1, 0), (2, 1)):                                            # those pages keep their contents
        p = int(table[0, h, col])
        for j in range(4):
            shape = cache.k.shape if j < 2 else (*cache.ks.shape, 4)
            want[j].view(shape)[p] = before[j].view(shape)[p]
    assert same(after, want)
    # indices outside the source, offsets outside idx
    cache.table_dev.copy_(good)
    idx = torch.tensor([[0, 25, -7, 3, 4]], dtype=torch.int32)
    offsets = torch.tensor([[0, 3, 4, 9, 9]], dtype=torch.int32)
    before = cache.bits()
    lens = cache.c.store(K.cuda(), V.cuda(), torch.zeros_like(start).cuda(), idx=idx.cuda(), offsets=offsets.cuda())
    assert cache.c.device_status() == B.CKV_EBOUNDS and cache.intact()
    rows = [[0, 25, -7], [3], [4], []]
    assert same(cache.bits(), expect_store(cache, before, K, V, lambda s, h: rows[h], torch.zeros_like(start)))
    assert lens.cpu().tolist() == [[3, 1, 1, 0]]
    assert cache.c.device_status() == 0                                        # read and cleared


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh,page,right", [(64, 16, False), (128, 64, True), (64, 128, True), (128, 32, False)])
def test_load_returns_the_stored_values(dtype, fmt, dh, page, right):
    lens = torch.tensor([[0, 1, 300], [37, 64, 129]], dtype=torch.int32)
    cache = Cache(nseq=2, Hq=3, Hkv=3, dh=dh, dtype=dtype, fmt=fmt, page=page, cols=-(-300 // page)).fill(lens, 5)
    if fmt == "plain":
        vals = [x.cpu() for x in (cache.k, cache.v)]
    else:
        vals = [(c.cpu().float() * s.cpu()[..., None]).to(R.DT[dtype]) for c, s in ((cache.k, cache.ks), (cache.v, cache.vs))]
    for n in (300, 311, 50):
        out = [Guarded((2, 3, n, dh), R.DT[dtype], fill=7.0) for _ in range(2)]
        cache.c.load(lens.cuda(), None, out[0].t, out[1].t, align_right=right)
        for o, v in zip(out, vals):
            want = torch.full((2, 3, n, dh), 7.0, dtype=R.DT[dtype])
            for s in range(2):
                for h in range(3):
                    L = int(lens[s, h])
                    m = min(L, n)
                    rows = R.head_rows(v, cache.table[s, h], L, page)
                    if m:
                        want[s, h, n - m if right else 0:][:m] = rows[L - m:] if right else rows[:m]
            assert torch.equal(o.t.cpu(), want) and o.intact()
    assert cache.c.device_status() == 0


def test_load_of_bad_lengths_and_pages():
    lens = torch.tensor([[10, 32]], dtype=torch.int32)
    cache = Cache(nseq=1, Hq=2, Hkv=2, dh=64, dtype="bf16", fmt="e4m3", page=16, cols=2,
                  flags=B.CKV_FLAG_DEBUG_CHECKS).fill(lens, 5)
    good, _ = cache.c.load(lens.cuda(), 40)
    assert cache.c.device_status() == 0
    got, _ = cache.c.load(torch.tensor([[-4, 99]], dtype=torch.int32, device="cuda"), 40)    # clipped to 0 and 32
    assert cache.c.device_status() == B.CKV_EBOUNDS
    assert bool((got[0, 0] == 0).all()) and torch.equal(got[0, 1], good[0, 1])
    cache.table_dev[0, 1, 0] = 12345
    got, _ = cache.c.load(lens.cuda(), 40)
    assert cache.c.device_status() == B.CKV_EBOUNDS
    assert bool((got[0, 1, :16] == 0).all()) and torch.equal(got[0, 1, 16:32], good[0, 1, 16:32])


# ---- decode ----------------------------------------------------------------------------------------------------------
def check_decode(cache, q, lens, got, scale=None):
    kv, vv = cache.values()
    scale = 1.0 / math.sqrt(cache.dh) if scale is None else scale
    out, lse, tol, tol_lse = R.decode(q, kv, vv, cache.table, lens, cache.page, scale, cache.fmt, cache.dtype, cache.vs)
    assert not bool(((got[0].cpu().double() - out).abs() > tol).any())
    empty = torch.isinf(lse)
    assert torch.equal(torch.isinf(got[1].cpu()), empty)
    assert not bool(((got[1].cpu().double() - lse).abs() > tol_lse)[~empty].any())


LENS = {
    "one": lambda n, h: torch.ones(n, h, dtype=torch.int32),
    "short": lambda n, h: torch.arange(n * h).view(n, h).remainder(19).to(torch.int32),
    "edges": lambda n, h: torch.tensor([15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 0])[
        torch.arange(n * h).remainder(16)].view(n, h).to(torch.int32),
    "ragged": lambda n, h: (torch.arange(n * h) * 211).remainder(1300).view(n, h).to(torch.int32),
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh,G,Hkv,nseq,page,lens", [
    (128, 4, 8, 1, 64, "ragged"), (64, 1, 2, 5, 16, "short"), (128, 8, 2, 8, 32, "edges"), (64, 5, 3, 6, 128, "edges"),
    (128, 1, 1, 1, 16, "one"), (64, 12, 2, 3, 64, "ragged"), (128, 16, 1, 2, 256, "ragged"), (128, 40, 1, 3, 16, "ragged"),
    (64, 32, 2, 2, 32, "short"), (128, 5, 8, 40, 16, "ragged")])
def test_decode(dtype, fmt, dh, G, Hkv, nseq, page, lens):
    lens = LENS[lens](nseq, Hkv)
    cols = max(1, -(-int(lens.max()) // page))
    cache = Cache(nseq=nseq, Hq=G * Hkv, Hkv=Hkv, dh=dh, dtype=dtype, fmt=fmt, page=page, cols=cols, seed=dh + G).fill(lens, G)
    q = (1.5 * torch.randn(nseq, G * Hkv, dh, generator=gen(G + 1))).to(R.DT[dtype])
    out, lse = Guarded((nseq, G * Hkv, dh), R.DT[dtype]), Guarded((nseq, G * Hkv), torch.float32)
    ws = Guarded((cache.c._ws_bytes,), torch.uint8)
    got = cache.c.attend(q.cuda(), lens.cuda(), out.t, lse.t, ws=ws.t)
    check_decode(cache, q, lens, got)
    assert out.intact() and lse.intact() and ws.intact() and cache.intact()
    assert cache.c.device_status() == 0
    assert B.criticalkv_last_path(cache.c.handle) & 384 == (128 if dtype == "bf16" else 256)
    again = cache.c.attend(q.cuda(), lens.cuda())                              # another workspace: the same bits
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    simt = PagedCache(Hq=G * Hkv, dtype=dtype, format=fmt, k_pages=cache.k, v_pages=cache.v, k_scale=cache.ks,
                      v_scale=cache.vs, page_table=cache.table_dev, flags=B.CKV_FLAG_FORCE_SIMT)
    check_decode(cache, q, lens, simt.attend(q.cuda(), lens.cuda()))
    assert B.criticalkv_last_path(simt.handle) & 256


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh,G,page,lens", [(128, 4, 16, "short"), (64, 8, 64, "edges"), (128, 16, 32, "edges"),
                                            (64, 3, 16, "one"), (128, 20, 128, "short")])
def test_decode_of_many_short_heads(fmt, dh, G, page, lens):
    """More heads than CTAs, each of a few rows: every warp works on its own.  One head is long and split over many."""
    nseq, Hkv = 60, 8
    lens = LENS[lens](nseq, Hkv)
    lens[31, 3] = 3001
    cols = -(-3001 // page)
    cache = Cache(nseq=nseq, Hq=G * Hkv, Hkv=Hkv, dh=dh, dtype="bf16", fmt=fmt, page=page, cols=cols).fill(lens, G)
    q = (1.5 * torch.randn(nseq, G * Hkv, dh, generator=gen(G + 1))).bfloat16()
    got = cache.c.attend(q.cuda(), lens.cuda())
    check_decode(cache, q, lens, got)
    again = cache.c.attend(q.cuda(), lens.cuda())
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    assert cache.c.device_status() == 0


@pytest.mark.parametrize("dtype,fmt", [("bf16", "plain"), ("bf16", "e4m3"), ("f32", "int8"), ("f32", "plain")])
@pytest.mark.parametrize("G", [1, 2, 3])
def test_decode_of_one_long_head(dtype, fmt, G):
    """All CTAs work on one KV head."""
    lens = torch.full((1, 1), 30011, dtype=torch.int32)
    cache = Cache(nseq=1, Hq=G, Hkv=1, dh=64, dtype=dtype, fmt=fmt, page=128, cols=235).fill(lens, 3)
    q = torch.randn(1, G, 64, generator=gen(8)).to(R.DT[dtype])
    check_decode(cache, q, lens, cache.c.attend(q.cuda(), lens.cuda()))


@pytest.mark.parametrize("dtype,fmt", [("bf16", "plain"), ("bf16", "e4m3"), ("f32", "int8"), ("f32", "plain")])
def test_decode_of_few_long_heads(dtype, fmt):
    """One long head next to short and empty ones: the long one is split over most CTAs and joined."""
    lens = torch.tensor([[20011, 3], [0, 1]], dtype=torch.int32)
    cache = Cache(nseq=2, Hq=8, Hkv=2, dh=128, dtype=dtype, fmt=fmt, page=64, cols=313).fill(lens, 3)
    q = torch.randn(2, 8, 128, generator=gen(8)).to(R.DT[dtype])
    check_decode(cache, q, lens, cache.c.attend(q.cuda(), lens.cuda()))


@pytest.mark.parametrize("dtype,fmt", [("bf16", "plain"), ("bf16", "e4m3"), ("f32", "int8"), ("f32", "plain")])
@pytest.mark.parametrize("dh,G,Hkv", [(128, 4, 2), (64, 16, 1), (64, 1, 7), (128, 9, 1), (64, 8, 25), (64, 20, 2)])
@pytest.mark.parametrize("rows", [16, 48, 130, 384, 760, 1300])
def test_decode_with_clusters_and_without(dtype, fmt, dh, G, Hkv, rows):
    """Few short heads: one launch, a CTA or a cluster a head; without clusters two launches but for the shortest."""
    cache = Cache(nseq=1, Hq=G * Hkv, Hkv=Hkv, dh=dh, dtype=dtype, fmt=fmt, page=16, cols=(rows + 15) // 16)
    full = torch.full((1, Hkv), rows, dtype=torch.int32)
    cache.fill(full, 2)
    apart = PagedCache(Hq=G * Hkv, dtype=dtype, format=fmt, k_pages=cache.k, v_pages=cache.v, k_scale=cache.ks,
                       v_scale=cache.vs, page_table=cache.table_dev, flags=B.CKV_FLAG_SELECT_NO_CLUSTER)
    q = torch.randn(1, G * Hkv, dh, generator=gen(3)).to(R.DT[dtype])
    for lens in (full, torch.zeros_like(full), (full - torch.arange(Hkv) * 7).clamp(min=0).to(torch.int32),
                 torch.arange(1, Hkv + 1, dtype=torch.int32).view(1, Hkv).clamp(max=rows)):
        for c, most in ((cache.c, 1 if rows < 1000 else 2), (apart, 1 if rows < 50 else 2)):
            before = B.criticalkv_launch_count(c.handle)
            got = c.attend(q.cuda(), lens.cuda())
            assert 1 <= B.criticalkv_launch_count(c.handle) - before <= most
            check_decode(cache, q, lens, got)


def test_decode_strided_queries_scale_and_shared_pages():
    lens = torch.tensor([[50, 20], [50, 33]], dtype=torch.int32)
    cache = Cache(nseq=2, Hq=8, Hkv=2, dh=64, dtype="bf16", fmt="plain", page=16, cols=4, scale=0.31).fill(lens, 3)
    cache.table[1, 0] = cache.table[0, 0]                                      # a prefix that two sequences share
    cache.table_dev.copy_(cache.table)
    both = torch.randn(2, 12, 64, generator=gen(8)).bfloat16()
    q = both.cuda()[:, 2:10]
    check_decode(cache, both[:, 2:10], lens, cache.c.attend(q, lens.cuda()), scale=0.31)


@pytest.mark.parametrize("dtype,fmt", [("bf16", "plain"), ("bf16", "e4m3"), ("bf16", "int8"), ("f32", "plain"), ("f32", "e4m3")])
def test_decode_with_values_of_very_different_size(dtype, fmt):
    """Value rows whose norms differ by many orders of magnitude, the large ones on rows with little weight."""
    lens = torch.tensor([[200, 97]], dtype=torch.int32)
    cache = Cache(nseq=1, Hq=4, Hkv=2, dh=64, dtype=dtype, fmt=fmt, page=32, cols=7).fill(lens, 3, spread=4.0)
    q = (3 * torch.randn(1, 4, 64, generator=gen(8))).to(R.DT[dtype])
    check_decode(cache, q, lens, cache.c.attend(q.cuda(), lens.cuda()))


def test_decode_large_and_tiny_queries():
    """bf16 queries far outside the range of a half (and its inverse), on 8-bit keys."""
    lens = torch.full((1, 1), 40, dtype=torch.int32)
    for fmt in ("e4m3", "int8"):
        for size in (2.0 ** 40, 2.0 ** -40, 0.0):
            cache = Cache(nseq=1, Hq=2, Hkv=1, dh=64, dtype="bf16", fmt=fmt, page=16, cols=3,
                          scale=1.0 / (8 * size) if size else 1.0).fill(lens, 3)
            q = (size * torch.randn(1, 2, 64, generator=gen(8))).bfloat16()
            check_decode(cache, q, lens, cache.c.attend(q.cuda(), lens.cuda()), scale=1.0 / (8 * size) if size else 1.0)


@pytest.mark.parametrize("scale", [0.0, 0.1, 0.13])     # scale * log2(e) rounds down and up
@pytest.mark.parametrize("dtype,fmt", [("bf16", "plain"), ("bf16", "e4m3"), ("bf16", "int8"), ("f32", "plain"), ("f32", "int8")])
def test_decode_infinities_and_nan(dtype, fmt, scale):
    """Rows with a NaN or an infinity make the heads that read them NaN, as in the formula, and no others; logits of
    -infinity have weight 0."""
    nan = math.nan
    lens = torch.tensor([[70, 70, 70, 70]], dtype=torch.int32)
    cache = Cache(nseq=1, Hq=4, Hkv=4, dh=64, dtype=dtype, fmt=fmt, page=16, cols=5, scale=scale).fill(lens, 3)
    scale = scale or 0.125
    q = torch.randn(1, 4, 64, generator=gen(8)).to(R.DT[dtype])
    page = cache.table[0, :, 2].long().tolist()
    where = (cache.v, cache.k) if fmt == "plain" else (cache.vs, cache.ks)
    where[0][page[1], 7] = nan                                                # a value row of head 1
    where[1][page[2], 9] = nan                                                # a key row of head 2
    out, lse = (x.cpu() for x in cache.c.attend(q.cuda(), lens.cuda()))
    assert bool(torch.isnan(out[0, 1]).all()) and bool(torch.isfinite(lse[0, 1]))
    assert bool(torch.isnan(out[0, 2]).all()) and bool(torch.isnan(lse[0, 2]))
    for h in (0, 3):
        assert bool(torch.isfinite(out[0, h]).all()) and bool(torch.isfinite(lse[0, h]))
    if fmt == "plain":
        # head 3: one key makes its logit -infinity; the result is the softmax over the others
        cache.k[page[3], 4, 0] = -math.inf if float(q[0, 3, 0]) > 0 else math.inf
        out, lse = (x.cpu().double() for x in cache.c.attend(q.cuda(), lens.cuda()))
        K, V = (R.head_rows(x, cache.table[0, 3], 70, 16) for x in cache.values())
        logit = K @ q[0, 3].double() * scale
        assert float(logit.min()) == -math.inf
        assert abs(float(lse[0, 3]) - float(torch.logsumexp(logit, 0))) < 1e-4
        want = torch.softmax(logit, 0) @ V
        assert float((out[0, 3] - want).abs().max()) < 0.02 * float(V.abs().max())
        # every logit of head 0 is -infinity: 0 / 0
        cache.k[cache.table[0, 0].long().tolist(), :, 0] = -math.inf if float(q[0, 0, 0]) > 0 else math.inf
        out, lse = (x.cpu() for x in cache.c.attend(q.cuda(), lens.cuda()))
        assert bool(torch.isnan(out[0, 0]).all()) and float(lse[0, 0]) == -math.inf


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_bad_lengths_and_pages(dtype):
    lens = torch.tensor([[48, 48, 30]], dtype=torch.int32)
    cache = Cache(nseq=1, Hq=6, Hkv=3, dh=64, dtype=dtype, fmt="plain", page=16, cols=3,
                  flags=B.CKV_FLAG_DEBUG_CHECKS).fill(lens, 3)
    q = torch.randn(1, 6, 64, generator=gen(8)).to(R.DT[dtype])
    good = cache.c.attend(q.cuda(), lens.cuda())
    assert cache.c.device_status() == 0
    check_decode(cache, q, lens, good)
    wild = torch.tensor([[2 ** 31 - 1, 49, -8]], dtype=torch.int32)            # clipped to 48, 48, 0
    got = cache.c.attend(q.cuda(), wild.cuda())
    assert cache.c.device_status() == B.CKV_EBOUNDS
    assert torch.equal(got[0][:, :4], good[0][:, :4])
    assert bool((got[0][:, 4:] == 0).all()) and bool(torch.isinf(got[1][:, 4:]).all())
    cache.table_dev[0, 0, 2], cache.table_dev[0, 1, 2] = -1, cache.k.shape[0]  # their last 16 rows are absent
    got = cache.c.attend(q.cuda(), lens.cuda())
    assert cache.c.device_status() == B.CKV_EBOUNDS
    check_decode(cache, q, torch.tensor([[32, 32, 30]], dtype=torch.int32), got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_of_a_head_without_any_page(dtype):
    lens = torch.tensor([[40, 40]], dtype=torch.int32)
    cache = Cache(nseq=1, Hq=2, Hkv=2, dh=64, dtype=dtype, fmt="e4m3", page=16, cols=3).fill(lens, 3)
    cache.table_dev[0, 0] = -1
    q = torch.randn(1, 2, 64, generator=gen(8)).to(R.DT[dtype])
    out, lse = (x.cpu() for x in cache.c.attend(q.cuda(), lens.cuda()))
    assert bool(torch.isnan(out[0, 0]).all()) and float(lse[0, 0]) == -math.inf
    assert bool(torch.isfinite(out[0, 1]).all()) and cache.c.device_status() == 0     # reported with debug checks only


def test_a_handle_is_shared_on_its_own_device_only():
    h = B.criticalkv_create(0)
    r = Rotary(dh=64, frequencies=rope_frequencies(64), device="cuda:0", handle=h)
    q = torch.ones(1, 1, 1, 64, device="cuda")
    pos = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    before = B.criticalkv_launch_count(h)
    r.rotate(q, None, pos)
    assert B.criticalkv_launch_count(h) == before + 1
    r.close()                                                     # does not destroy what it does not own
    assert B.criticalkv_launch_count(h) == before + 1
    h.device = 1
    with pytest.raises(ValueError):
        Rotary(dh=64, frequencies=rope_frequencies(64), device="cuda:0", handle=h)
    B.criticalkv_destroy(h)


def test_compact_into_follows_the_stream_of_the_session():
    """With a side stream current, a session without a stream argument works on the default stream, the store with it."""
    g = gen(21)
    Hq, Hkv, dh, dm, n, w = 4, 2, 64, 64, 4000, 8
    Qw, K, V, WO = (torch.randn(*s, generator=g).bfloat16().cuda() for s in (
        (1, Hq, w, dh), (1, Hkv, n, dh), (1, Hkv, n, dh), (1, Hq, dh, dm)))
    kw = dict(nb=1, Hq=Hq, Hkv=Hkv, dh=dh, dm=dm, n=n, w=w, pool_k=3, dtype="bf16", budget_mode="uniform", budget=700)
    s = CompressionSession(**kw)
    cache = PagedCache.allocate(nseq=1, Hq=Hq, Hkv=Hkv, dh=dh, dtype="bf16", rows=n)
    start = cache.new_lengths()
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        s.compress(Qw, K, V, WO)
        lens = s.compact_into(cache, K, V, start)
    torch.cuda.synchronize()
    got, _ = cache.load(lens, 700)
    assert torch.equal(got[0].reshape(-1, dh), s.K_out[0])


def test_empty_batches():
    cache = Cache(nseq=0, Hq=4, Hkv=2, dh=64, dtype="bf16", fmt="e4m3", page=16, cols=1)
    lens = torch.zeros(0, 2, dtype=torch.int32, device="cuda")
    q = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    K = torch.zeros(0, 2, 3, 64, dtype=torch.bfloat16, device="cuda")
    assert cache.c.attend(q, lens)[0].shape == q.shape
    assert cache.c.store(K, K, lens).shape == lens.shape and cache.c.load(lens, 5)[0].shape == (0, 2, 5, 64)
    cache = Cache(nseq=1, Hq=4, Hkv=2, dh=64, dtype="bf16", fmt="e4m3", page=16, cols=1)
    lens = torch.tensor([[3, 4]], dtype=torch.int32, device="cuda")
    none = torch.zeros(1, 2, 0, 64, dtype=torch.bfloat16, device="cuda")
    assert torch.equal(cache.c.store(none, none, lens), lens)
    assert cache.c.load(lens, 0)[0].shape == (1, 2, 0, 64)
    some = torch.zeros(1, 2, 5, 64, dtype=torch.bfloat16, device="cuda")
    assert torch.equal(cache.c.store(some, some, lens, idx=torch.zeros(1, 0, dtype=torch.int32, device="cuda"),
                                     offsets=torch.zeros(1, 3, dtype=torch.int32, device="cuda")), lens)


@pytest.mark.parametrize("dtype,fmt", [("bf16", "plain"), ("bf16", "e4m3"), ("f32", "int8")])
def test_pages_beyond_4_gigabytes(dtype, fmt):
    """Page ids whose byte (and for plain pages element) offsets pass 32 bits."""
    page, dh = 256, 128
    size = {"plain": 2 if dtype == "bf16" else 4}.get(fmt, 1)
    n = (2 ** 32 // size) // (page * dh) * (1 if fmt != "plain" else 2) + 8    # beyond 2^32 bytes, 2^32 elements if plain
    code = R.CODE.get(fmt, R.DT[dtype])
    raw = torch.uint8 if fmt != "plain" else code
    k, v = (torch.empty((n, page, dh), dtype=raw, device="cuda").view(code) for _ in range(2))
    ks, vs = (torch.empty((n, page), device="cuda") if fmt != "plain" else None for _ in range(2))
    table = torch.tensor([[[n - 1, 0, n - 2]]], dtype=torch.int32, device="cuda")
    c = PagedCache(Hq=4, dtype=dtype, format=fmt, k_pages=k, v_pages=v, k_scale=ks, v_scale=vs, page_table=table)
    small_table = torch.tensor([[[0, 1, 2]]], dtype=torch.int32, device="cuda")
    sk, sv = (torch.zeros((3, page, dh), dtype=raw, device="cuda").view(code) for _ in range(2))
    sks, svs = (torch.zeros((3, page), device="cuda") if fmt != "plain" else None for _ in range(2))
    small = PagedCache(Hq=4, dtype=dtype, format=fmt, k_pages=sk, v_pages=sv, k_scale=sks, v_scale=svs, page_table=small_table)
    g = gen(5)
    K, V = (torch.randn(1, 1, 700, dh, generator=g).to(R.DT[dtype]).cuda() for _ in range(2))
    q = torch.randn(1, 4, dh, generator=g).to(R.DT[dtype]).cuda()
    zero = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    for x in (c, small):
        x.store(K, V, zero)
    lens = zero + 700
    for a, b in zip(c.load(lens, 700) + c.attend(q, lens), small.load(lens, 700) + small.attend(q, lens)):
        assert torch.equal(a, b)


def test_calls_in_a_captured_graph_and_on_another_stream():
    """A decode step (rotate, store, attend) captured once and replayed: every replay appends a token; the same steps
    on a side stream give the same bits."""
    nseq, Hq, Hkv, dh, steps = 3, 8, 2, 64, 5

    def fresh():
        cache = PagedCache.allocate(nseq=nseq, Hq=Hq, Hkv=Hkv, dh=dh, dtype="bf16", rows=200, format="e4m3", page_size=16)
        g = gen(3)
        lens = torch.tensor([[100, 33], [0, 1], [17, 150]], dtype=torch.int32, device="cuda")
        K, V = (torch.randn(nseq, Hkv, 150, dh, generator=g).bfloat16().cuda() for _ in range(2))
        cache.store(K, V, cache.new_lengths())
        return cache, lens

    rotary = Rotary(dh=dh, frequencies=rope_frequencies(dh), device="cuda:0")
    g = gen(7)
    tokens = [tuple(torch.randn(nseq, H, 1, dh, generator=g).bfloat16().cuda() for H in (Hq, Hkv, Hkv)) for _ in range(steps)]
    pos0 = torch.full((nseq, 1), 5000, dtype=torch.int32, device="cuda")

    def step(cache, q, k, v, pos, lens, stream=None):
        qr, kr = rotary.rotate(q, k, pos, stream=stream)
        cache.store(kr, v, lens, lens, stream=stream)
        return cache.attend(qr[:, :, 0], lens, stream=stream)

    cache, lens = fresh()
    plain = []
    for i, (q, k, v) in enumerate(tokens):
        plain.append([x.clone() for x in step(cache, q, k, v, pos0 + i, lens)])
    assert torch.equal(lens.cpu(), torch.tensor([[105, 38], [5, 6], [22, 155]], dtype=torch.int32))

    cache, lens = fresh()
    cache.workspace()
    q, k, v = (torch.empty_like(x) for x in tokens[0])
    pos = pos0.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step(cache, q, k, v, pos, lens)
    for i, t in enumerate(tokens):
        for dst, src in zip((q, k, v), t):
            dst.copy_(src)
        pos.copy_(pos0 + i)
        graph.replay()
        assert torch.equal(out, plain[i][0]) and torch.equal(lse, plain[i][1])

    cache, lens = fresh()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = [step(cache, q, k, v, pos0 + i, lens, stream=side) for i, (q, k, v) in enumerate(tokens)]
    side.synchronize()
    for a, b in zip(got, plain):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_two_calls_at_once_with_workspaces_of_their_own():
    lens = torch.tensor([[5000, 700]], dtype=torch.int32)
    cache = Cache(nseq=1, Hq=8, Hkv=2, dh=128, dtype="bf16", fmt="plain", page=64, cols=79).fill(lens, 3)
    qs = [torch.randn(1, 8, 128, generator=gen(i)).bfloat16().cuda() for i in range(2)]
    dev = lens.cuda()
    want = [cache.c.attend(q, dev) for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    spaces = [torch.empty_like(cache.c.workspace()) for _ in qs]
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        got.append([cache.c.attend(q, dev, ws=w, stream=s) for q, w, s in zip(qs, spaces, streams)])
    torch.cuda.synchronize()
    for pair in got:
        for a, b in zip(pair, want):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_cache_refuses_bad_tensors():
    cache = Cache(nseq=2, Hq=4, Hkv=2, dh=64, dtype="bf16", fmt="e4m3", page=16, cols=2)
    c = cache.c
    lens = torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    K = torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    calls = [
        lambda: c.store(K.float(), K, lens), lambda: c.store(K, K[:, :, :2], lens), lambda: c.store(K.cpu(), K.cpu(), lens),
        lambda: c.store(K, K, lens.long()), lambda: c.store(K, K, lens[:1]), lambda: c.store(K, K, lens.t()[:, :1]),
        lambda: c.store(K, K, lens, idx=lens), lambda: c.store(K, K, lens, counts=lens),
        lambda: c.store(K, K.transpose(1, 2).contiguous().transpose(1, 2), lens),
        lambda: c.load(lens), lambda: c.load(lens, 3, K, None), lambda: c.load(lens, 4, K, K.clone()),
        lambda: c.load(lens, None, K.float(), K.float()),
        lambda: c.attend(q.float(), lens), lambda: c.attend(q[:, :2], lens), lambda: c.attend(q, lens.cpu()),
        lambda: c.attend(q, lens, out=q[:, :2]), lambda: c.attend(q, lens, lse=torch.zeros(2, 4, device="cuda").double()),
        lambda: PagedCache(Hq=4, dtype="bf16", format="e4m3", k_pages=cache.k, v_pages=cache.v, page_table=cache.table_dev),
        lambda: PagedCache(Hq=4, dtype="bf16", format="int4", k_pages=cache.k, v_pages=cache.v, page_table=cache.table_dev),
        lambda: PagedCache(Hq=4, dtype="bf16", k_pages=cache.k, v_pages=cache.v, page_table=cache.table_dev),
        lambda: PagedCache(Hq=4, dtype="bf16", format="e4m3", k_pages=cache.k, v_pages=cache.v, k_scale=cache.ks,
                           v_scale=cache.vs, page_table=cache.table),
    ]
    for f in calls:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(B.CriticalKVError):
        c.attend(q, lens, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(B.CriticalKVError):                                     # 3 query heads on 2 KV heads
        PagedCache(Hq=3, dtype="bf16", format="e4m3", k_pages=cache.k, v_pages=cache.v, k_scale=cache.ks,
                   v_scale=cache.vs, page_table=cache.table_dev)


# ---- the operators together, as a serving loop uses them --------------------------------------------------------------
@pytest.mark.parametrize("mode,fmt", [("adaptive", "plain"), ("uniform", "e4m3"), ("adaptive", "int8")])
def test_compress_store_and_decode(mode, fmt):
    """Prefill compression -> selected rows into the paged cache -> new tokens rotated, appended and attended."""
    Hq, Hkv, dh, dm, n, w = 8, 4, 64, 128, 500, 16
    g = gen(11)
    nb = 2
    Qw, K, V, WO = (torch.randn(*s, generator=g).bfloat16().cuda() for s in (
        (nb, Hq, w, dh), (nb, Hkv, n, dh), (nb, Hkv, n, dh), (nb, Hq, dh, dm)))
    budget = 120 if mode == "uniform" else 480
    s = CompressionSession(nb=nb, Hq=Hq, Hkv=Hkv, dh=dh, dm=dm, n=n, w=w, pool_k=5, dtype="bf16", budget_mode=mode,
                           budget=budget)
    s.compress(Qw, K, V, WO)
    cache = PagedCache.allocate(nseq=nb, Hq=Hq, Hkv=Hkv, dh=dh, dtype="bf16", rows=n + 8, format=fmt, page_size=16)
    lens = s.compact_into(cache, K, V, cache.new_lengths())
    off = s.offsets.cpu()
    assert torch.equal(lens.cpu(), off.diff(dim=1))
    # what the cache holds is what compact gathered (through the format's rounding)
    Kl, Vl = cache.load(lens, n)
    for b in range(nb):
        for h in range(Hkv):
            lo, hi = int(off[b, h]), int(off[b, h + 1])
            for got, kept in ((Kl, s.K_out), (Vl, s.V_out)):
                rows = kept[b, lo:hi].cpu()
                if fmt != "plain":
                    code, scale = R.quantise(rows, fmt)
                    rows = (code.float() * scale[:, None]).bfloat16()
                assert torch.equal(got[b, h, :hi - lo].cpu(), rows)
    rotary = Rotary(dh=dh, frequencies=rope_frequencies(dh), device="cuda:0")
    for t in range(3):
        q, k, v = (torch.randn(nb, H, 1, dh, generator=g).bfloat16().cuda() for H in (Hq, Hkv, Hkv))
        qr, kr = rotary.rotate(q, k, torch.full((nb, 1), n + t, dtype=torch.int32, device="cuda"))
        lens = cache.store(kr, v, lens, lens)
        out, lse = cache.attend(qr[:, :, 0], lens)
        kv, vv = R.stored(cache.k_pages, cache.k_scale, fmt), R.stored(cache.v_pages, cache.v_scale, fmt)
        want, want_lse, tol, tol_lse = R.decode(qr[:, :, 0].cpu(), kv, vv, cache.page_table.cpu(), lens.cpu(), 16, 0.125, fmt,
                                                "bf16", cache.v_scale)
        assert not bool(((out.cpu().double() - want).abs() > tol).any())
        assert not bool(((lse.cpu().double() - want_lse).abs() > tol_lse).any())
    assert cache.device_status() == 0


@pytest.mark.parametrize("mode", ["uniform", "adaptive"])
def test_chunked_prefill_into_a_cache_and_back(mode):
    """Chunked prefill ends in a paged cache; read back right-aligned it is the ragged input of another compression."""
    Hq, Hkv, dh, dm, w = 4, 2, 64, 64, 8
    g = gen(12)
    ch = ChunkedPrefillCompressor(Hq=Hq, Hkv=Hkv, dh=dh, dm=dm, w=w, pool_k=3, dtype="f32", budget_mode=mode)
    WO = torch.randn(Hq, dh, dm, generator=g).cuda()
    for n in (90, 70):
        ch.step(torch.randn(Hq, w, dh, generator=g).cuda(), torch.randn(Hkv, n, dh, generator=g).cuda(),
                torch.randn(Hkv, n, dh, generator=g).cuda(), WO, 60 if mode == "uniform" else 120)
    cache = PagedCache.allocate(nseq=1, Hq=Hq, Hkv=Hkv, dh=dh, dtype="f32", rows=200, page_size=32)
    lens = ch.to_cache(cache)
    assert lens.cpu().tolist() == [[int(k.shape[0]) for k in ch.K]]
    n = int(lens.max())
    K, V = cache.load(lens, n, align_right=True)
    for h in range(Hkv):
        m = int(lens[0, h])
        assert torch.equal(K[0, h, n - m:], ch.K[h]) and torch.equal(V[0, h, n - m:], ch.V[h])
        assert bool((K[0, h, :n - m] == 0).all())
    valid = (n - lens).contiguous()
    s = CompressionSession(nb=1, Hq=Hq, Hkv=Hkv, dh=dh, dm=dm, n=n, w=w, pool_k=3, dtype="f32", budget_mode="adaptive",
                           budget=50, valid_from=valid)
    s.compress(torch.randn(1, Hq, w, dh, generator=g).cuda(), K, V, WO[None])
    off = s.offsets[0].cpu()
    assert int(off[-1]) == 50
    for h in range(Hkv):
        assert int(s.idx[0, int(off[h]):int(off[h + 1])].min()) >= int(valid[0, h])


@pytest.mark.parametrize("mode", ["uniform", "adaptive"])
def test_to_cache_on_a_stream_of_its_own(mode):
    """All that to_cache launches goes to the stream it is given: a busy current stream does not hold any of it back."""
    g = gen(14)
    Hq, Hkv, dh, dm, w, n = 4, 2, 64, 64, 8, 90
    ch = ChunkedPrefillCompressor(Hq=Hq, Hkv=Hkv, dh=dh, dm=dm, w=w, pool_k=3, dtype="bf16", budget_mode=mode)
    ch.step(*(torch.randn(*s, generator=g).bfloat16().cuda() for s in (
        (Hq, w, dh), (Hkv, n, dh), (Hkv, n, dh), (Hq, dh, dm))), 40 if mode == "uniform" else 80)
    cache = PagedCache.allocate(nseq=1, Hq=Hq, Hkv=Hkv, dh=dh, dtype="bf16", rows=100)
    blocks = [torch.full((1, Hkv), 77, dtype=torch.int32, device="cuda") for _ in range(64)]
    del blocks                                       # what the allocator hands out next holds a wrong length
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(400_000_000)                   # about 0.2 s
    lens = ch.to_cache(cache, stream=side)
    side.synchronize()
    assert not torch.cuda.default_stream().query()   # still asleep
    torch.cuda.synchronize()
    assert lens.cpu().tolist() == [[int(k.shape[0]) for k in ch.K]]
    K, V = cache.load(lens, int(lens.max()))
    for h in range(Hkv):
        m = int(lens[0, h])
        assert torch.equal(K[0, h, :m], ch.K[h]) and torch.equal(V[0, h, :m], ch.V[h])
