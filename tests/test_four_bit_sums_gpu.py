"""float32 queries on 4-bit pages: sums that are rounded and not cut off, shown where a chain of cut-off sums is far outside."""
import math

import pytest
import torch

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
