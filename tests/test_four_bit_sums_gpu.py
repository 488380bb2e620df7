"""float32 queries on 4-bit pages: sums that are rounded and not cut off, shown where a chain of cut-off sums is far outside."""
import math

import pytest
import torch

import four_bit as F
from paper_2502_03805_b200 import PagedCache
from paper_2502_03805_b200 import binding as B
from test_cache_gpu import gen

pytestmark = pytest.mark.gpu
STEP = 2.0 ** -23                 # of float32, relative; a rounding is off by half of it at most, a sum cut off by one


@pytest.mark.parametrize("dh,G,rows", [(128, 1, 100000), (128, 4, 100000), (128, 8, 100000), (64, 3, 100000), (64, 8, 100000),
                                       (128, 2, 400000)])
def test_long_heads_with_values_of_one_sign(dh, G, rows):
    """Queries of zeros: every weight is 1 and the result the mean of the values, which lie between 1/2 and 3/2.

    56 x 8 heads on the same pages, so that a CTA has a whole head or two halves and a warp a chain of rows / 64 tiles of 16
    rows.  A tile's sum is exact but for 4 STEP (the matrix instructions cut off, two of them a tile at most, in two parts each
    perhaps).  The additions of the tiles are rounded: each is off by at most half a step of the sum so far, independently
    and to both sides, a standard deviation of STEP / sqrt(12), so sqrt(tiles / 12) STEP of the result together (eight of them
    allowed: 5e5 results).  A weight times its row's scale is two halves (2^-22); 16 more roundings of half a step: weight and scale,
    references (three, and three when they move once), four warps, three parts, the sum's reciprocal and the result.
    In one chain of cut-off sums the results are low by about 0.36 STEP a tile: 6e-5 and 2.4e-4."""
    nseq, Hkv = 56, 8
    one = PagedCache.allocate(nseq=1, Hq=1, Hkv=1, dh=dh, dtype="f32", rows=rows, format="e2m1")
    K = torch.randn(1, 1, rows, dh, generator=gen(1)).cuda()
    V = (0.5 + torch.rand(1, 1, rows, dh, generator=gen(2))).cuda()
    length = one.store(K, V, one.new_lengths())
    mean = one.load(length, rows)[1][0, 0].double().mean(0)        # code times group scale times scale: one rounding of half a step
    c = PagedCache(Hq=G * Hkv, dtype="f32", format="e2m1", k_pages=one.k_pages, v_pages=one.v_pages, k_scale=one.k_scale,
                   v_scale=one.v_scale, k_group_scale=one.k_group_scale, v_group_scale=one.v_group_scale,
                   page_table=one.page_table.expand(nseq, Hkv, -1).contiguous())
    lens = torch.full((nseq, Hkv), rows, dtype=torch.int32, device="cuda")
    out, lse = c.attend(torch.zeros(nseq, G * Hkv, dh, device="cuda"), lens)
    assert B.criticalkv_last_path(c.handle) & 384 == 128
    tol = 8 * math.sqrt(rows / 64 / 12) * STEP + 4 * STEP + 2.0 ** -22 + 17 * STEP / 2
    assert bool(((out.double() - mean).abs() <= tol * mean).all())
    # the sum of the weights is exact; its logarithm, the product and the product's factor
    assert bool(((lse.double() - math.log(rows)).abs() <= 2 * STEP * math.log(rows)).all())


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("G", [1, 5])
@pytest.mark.parametrize("place", [0, 17, 63])
def test_logits_of_one_large_and_many_small_products(dh, G, place):
    """One product of 1 and dh - 1 of d each, sixteen of which (a matrix instruction's) are 0.9 steps of 1: a chain of cut-off
    sums loses all of them, 127 d or 63 d.

    The sum begins anew with every two instructions, so the 31 d beside the large product may be lost, and up to three
    additions of such sums are rounded (the second halves of these queries are zero).  The logit's factor, scale * log2(e), is 1
    to within 2^-28, the sum of the weights 1; the logarithm's factor 0.693 is off by 2^-28 of it and the result by a rounding."""
    cache = F.FourBit(nseq=1, Hq=G, Hkv=1, dh=dh, dtype="f32", page=16, cols=1, scale=math.log(2.0))
    page = int(cache.table[0, 0, 0])
    for code, group, scale in cache.parts():
        code[page, 0], group.view(torch.uint8)[page, 0], scale[page, 0] = 0x22, 0x38, 1.0          # a row of ones
    assert bool((cache.values()[0][page, 0] == 1).all())
    d = round(0.9 * 2048) / 2048 * 2.0 ** -27
    q = torch.full((1, G, dh), d)
    q[0, :, place] = 1.0
    out, lse = cache.c.attend(q.cuda(), torch.ones(1, 1, dtype=torch.int32, device="cuda"))
    ln2 = float(torch.tensor(math.log(2.0), dtype=torch.float32))
    want = ln2 * (1 + (dh - 1) * d)
    tol = ln2 * (31 * d + (dh // 32 - 1) * STEP / 2 + 2 * 2.0 ** -28) + 2.0 ** -25
    assert tol < 0.8 * ln2 * (dh - 1) * d                          # what the chain loses is far outside
    assert bool(((lse.double().cpu() - want).abs() <= tol).all())
    assert bool((out.cpu() == 1).all())
