"""Decode attention and rotary positions against 64 bits with comparisons that a NaN fails, every kernel held to its own
bound (float32 queries to float32 weights)."""
import math

import pytest
import torch

import cache_ref as R
import decode_bounds as D
from paper_2502_03805_b200 import PagedCache, Rotary
from paper_2502_03805_b200 import binding as B
from paper_2502_03805_b200 import rope_frequencies
from test_cache_gpu import FORMATS, LENS, Cache, gen, rope_tol

pytestmark = pytest.mark.gpu
MOVES = 16        # running maxima of a warp over a few thousand rows in random order: about ln n, and the joins


def check(cache, q, lens, c=None, kernel=None, scale=None, given=None):
    """attend on `c` (the cache's own object) and the comparison; `given`: lengths to pass where they differ from `lens`."""
    c = cache.c if c is None else c
    q_dev, lens_dev = q.cuda(), (lens if given is None else given).cuda()
    got = c.attend(q_dev, lens_dev)
    kernel = kernel or ("tensor" if cache.dtype == "bf16" else "cuda")
    assert B.criticalkv_last_path(c.handle) & 384 == (128 if kernel == "tensor" else 256)
    kv, vv = cache.values()
    want = D.decode(q, kv, vv, cache.table, lens, cache.page, 1.0 / math.sqrt(cache.dh) if scale is None else scale, cache.fmt,
                    cache.dtype, kernel, cache.vs, MOVES)
    D.check(got, want, lens, q.shape[1] // cache.Hkv)
    return got


def other(cache, Hq, flags):
    return PagedCache(Hq=Hq, dtype=cache.dtype, format=cache.fmt, k_pages=cache.k, v_pages=cache.v, k_scale=cache.ks,
                      v_scale=cache.vs, page_table=cache.table_dev, flags=flags)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh,G,Hkv,nseq,page,lens", [
    (128, 4, 8, 1, 64, "ragged"), (64, 1, 2, 5, 16, "short"), (128, 8, 2, 8, 32, "edges"), (64, 5, 3, 6, 128, "edges"),
    (128, 1, 1, 1, 16, "one"), (64, 12, 2, 3, 64, "ragged"), (128, 16, 1, 2, 256, "ragged"), (128, 40, 1, 3, 16, "ragged"),
    (64, 32, 2, 2, 32, "short"), (128, 5, 8, 40, 16, "ragged")])
@pytest.mark.parametrize("size", [0.1, 1.5])      # small queries: logits whose own errors do not hide those of the weights
def test_shapes(dtype, fmt, dh, G, Hkv, nseq, page, lens, size):
    lens = LENS[lens](nseq, Hkv)
    cols = max(1, -(-int(lens.max()) // page))
    cache = Cache(nseq=nseq, Hq=G * Hkv, Hkv=Hkv, dh=dh, dtype=dtype, fmt=fmt, page=page, cols=cols, seed=dh + G).fill(lens, G)
    q = (size * torch.randn(nseq, G * Hkv, dh, generator=gen(G + 1))).to(R.DT[dtype])
    check(cache, q, lens)
    check(cache, q, lens, other(cache, G * Hkv, B.CKV_FLAG_FORCE_SIMT), "cuda")


@pytest.mark.parametrize("dtype,fmt", [("bf16", "plain"), ("bf16", "e4m3"), ("f32", "int8"), ("f32", "plain")])
@pytest.mark.parametrize("G,nseq,Hkv,lens", [(1, 1, 1, [[30011]]), (3, 1, 1, [[30011]]), (4, 2, 2, [[20011, 3], [0, 1]]),
                                             (2, 3, 3, [[7000, 1, 64], [0, 9000, 129], [12000, 65, 63]])])
def test_long_heads(dtype, fmt, G, nseq, Hkv, lens):
    lens = torch.tensor(lens, dtype=torch.int32)
    cache = Cache(nseq=nseq, Hq=G * Hkv, Hkv=Hkv, dh=64, dtype=dtype, fmt=fmt, page=128, cols=235).fill(lens, 3)
    check(cache, torch.randn(nseq, G * Hkv, 64, generator=gen(8)).to(R.DT[dtype]), lens)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh,G,page,lens", [(128, 4, 16, "short"), (64, 8, 64, "edges"), (128, 16, 32, "edges")])
def test_many_short_heads_and_a_long_one(fmt, dh, G, page, lens):
    nseq, Hkv = 60, 8
    lens = LENS[lens](nseq, Hkv)
    lens[31, 3] = 3001
    cache = Cache(nseq=nseq, Hq=G * Hkv, Hkv=Hkv, dh=dh, dtype="bf16", fmt=fmt, page=page, cols=-(-3001 // page)).fill(lens, G)
    check(cache, (1.5 * torch.randn(nseq, G * Hkv, dh, generator=gen(G + 1))).bfloat16(), lens)


@pytest.mark.parametrize("dtype,fmt", [("bf16", "plain"), ("bf16", "e4m3"), ("f32", "int8"), ("f32", "plain")])
@pytest.mark.parametrize("dh,G,Hkv", [(128, 4, 2), (64, 16, 1), (64, 8, 25)])
@pytest.mark.parametrize("rows", [48, 384, 1300])
def test_clusters_and_none(dtype, fmt, dh, G, Hkv, rows):
    cache = Cache(nseq=1, Hq=G * Hkv, Hkv=Hkv, dh=dh, dtype=dtype, fmt=fmt, page=16, cols=(rows + 15) // 16)
    full = torch.full((1, Hkv), rows, dtype=torch.int32)
    cache.fill(full, 2)
    apart = other(cache, G * Hkv, B.CKV_FLAG_SELECT_NO_CLUSTER)
    q = torch.randn(1, G * Hkv, dh, generator=gen(3)).to(R.DT[dtype])
    for lens in (full, torch.zeros_like(full), (full - torch.arange(Hkv) * 7).clamp(min=0).to(torch.int32)):
        check(cache, q, lens)
        check(cache, q, lens, apart)


@pytest.mark.parametrize("dtype,fmt", [("bf16", "plain"), ("bf16", "e4m3"), ("bf16", "int8"), ("f32", "plain"), ("f32", "e4m3")])
def test_values_of_very_different_size(dtype, fmt):
    lens = torch.tensor([[200, 97]], dtype=torch.int32)
    cache = Cache(nseq=1, Hq=4, Hkv=2, dh=64, dtype=dtype, fmt=fmt, page=32, cols=7).fill(lens, 3, spread=4.0)
    check(cache, (3 * torch.randn(1, 4, 64, generator=gen(8))).to(R.DT[dtype]), lens)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("size", [2.0 ** 40, 2.0 ** -40, 0.0])
def test_large_and_tiny_queries(fmt, size):
    lens = torch.full((1, 1), 40, dtype=torch.int32)
    scale = 1.0 / (8 * size) if size else 1.0
    cache = Cache(nseq=1, Hq=2, Hkv=1, dh=64, dtype="bf16", fmt=fmt, page=16, cols=3, scale=scale).fill(lens, 3)
    check(cache, (size * torch.randn(1, 2, 64, generator=gen(8))).bfloat16(), lens, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_absent_pages_and_wild_lengths(dtype):
    lens = torch.tensor([[48, 48, 30]], dtype=torch.int32)
    cache = Cache(nseq=1, Hq=6, Hkv=3, dh=64, dtype=dtype, fmt="plain", page=16, cols=3,
                  flags=B.CKV_FLAG_DEBUG_CHECKS).fill(lens, 3)
    q = torch.randn(1, 6, 64, generator=gen(8)).to(R.DT[dtype])
    check(cache, q, lens)
    check(cache, q, torch.tensor([[48, 48, 0]], dtype=torch.int32),
          given=torch.tensor([[2 ** 31 - 1, 49, -8]], dtype=torch.int32))
    assert cache.c.device_status() == B.CKV_EBOUNDS
    cache.table_dev[0, 0, 2], cache.table_dev[0, 1, 2] = -1, cache.k.shape[0]
    check(cache, q, torch.tensor([[32, 32, 30]], dtype=torch.int32), given=lens)
    assert cache.c.device_status() == B.CKV_EBOUNDS


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("nseq,Hq,Hk,T,dh,rot,factor", [
    (1, 32, 8, 1, 128, 128, 1.0), (3, 5, 1, 17, 64, 64, 1.25), (1, 2, 2, 100, 64, 6, 1.0), (7, 4, 4, 1, 64, 20, 1.0),
    (1, 3, 1, 5, 256, 256, 1.0), (2, 9, 1, 70, 24, 16, 0.75), (3, 70, 1, 2, 128, 32, 1.0)])
def test_rope(dtype, layout, nseq, Hq, Hk, T, dh, rot, factor):
    g = gen(1)
    xs = [torch.randn(nseq, H, T, dh, generator=g).to(R.DT[dtype]) for H in (Hq, Hk)]
    pos = torch.randint(0, 140000, (nseq, T), generator=g, dtype=torch.int32)
    freq = rope_frequencies(rot, 500000.0)
    r = Rotary(dh=dh, frequencies=freq, layout=layout, factor=factor, device="cuda:0")
    for got, x in zip(r.rotate(xs[0].cuda(), xs[1].cuda(), pos.cuda()), xs):
        want = R.rope(x, pos, freq, layout, factor)
        assert bool(((got.cpu().double() - want).abs() <= rope_tol(x, want, layout, freq.numel(), dtype, factor)).all())
        assert torch.equal(got.cpu()[..., rot:], x[..., rot:])
