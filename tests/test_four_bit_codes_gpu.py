"""Every byte at every place of a 4-bit row, through each way of reading it: load, both products of both decode kernels, summaries."""

import pytest
import torch

import cache_ref as R
import four_bit as F
from paper_2502_03805_b200 import binding as B
from test_cache_gpu import gen
from test_pages_gpu import float32_keys, summary_of

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -24                 # half a step of float32, relative


@pytest.fixture(scope="module", params=[(64, "f32"), (64, "bf16"), (128, "f32"), (128, "bf16")], ids=str)
def rows(request):
    """256 sequences of one row; byte j of row s is (s + 37 j) mod 256.  Values of K are read back by queries of one element."""
    dh, dtype = request.param
    cache = F.FourBit(nseq=256, Hq=dh, Hkv=1, dh=dh, dtype=dtype, page=16, cols=1)
    s = torch.arange(256)
    g = gen(dh)
    for i, (code, group, scale) in enumerate(cache.parts()):
        page = cache.table[:, 0, 0].long().cuda()
        code[page, 0] = ((s[:, None] + 37 * torch.arange(dh // 2) + 101 * i) % 256).to(torch.uint8).cuda()
        group.view(torch.uint8)[page, 0] = torch.randint(0, 0x7f, (256, dh // 16), generator=g, dtype=torch.uint8).cuda()   # no NaN
        scale[page, 0] = torch.exp(torch.randn(256, generator=g)).cuda()
    K, V = (x[cache.table[:, 0, 0].long(), 0] for x in cache.values())
    return cache, K, V


def test_load(rows):
    cache, K, V = rows
    got = cache.c.load(torch.ones(256, 1, dtype=torch.int32, device="cuda"), 1)
    for x, want in zip(got, (K, V)):
        assert torch.equal(x[:, 0, 0].cpu(), want.float().to(R.DT[cache.dtype]))      # one rounding a step


@pytest.mark.parametrize("kernel", ["tensor", "cuda"])
@pytest.mark.parametrize("G", [1, 8, 16, 0])
def test_decode(rows, kernel, G):
    """One row a sequence: the result is the row of V, and the logit of a query of one element an element of K."""
    cache, K, V = rows
    dh, lens = cache.dh, torch.ones(256, 1, dtype=torch.int32, device="cuda")
    G = G or dh
    cache.Hq = G
    c = cache.other(flags=B.CKV_FLAG_FORCE_SIMT if kernel == "cuda" else 0, scale=1.0)
    for first in range(0, dh, G):
        q = torch.eye(dh)[first:first + G].to(R.DT[cache.dtype]).repeat(256, 1, 1)
        out, lse = (x.cpu().double() for x in c.attend(q.cuda(), lens))
        # a weight times a scale is two halves (2^-22) or a float, and twelve roundings or cut-off sums (two halves of a step)
        assert bool(((out - V[:, None]).abs() <= V[:, None].abs() * (2.0 ** -22 + 24 * HALF + R.HALF_STEP[cache.dtype])).all())
        # exact products; the row's scale, the logit's factor and its product, the logarithm's factor and the result
        want = K[:, first:first + G]
        assert bool(((lse - want).abs() <= want.abs() * 8 * HALF).all())


def test_summaries(rows):
    cache, K, V = rows
    summary = cache.c.summarise(cache.c.new_summary(), torch.ones(256, 1, dtype=torch.int32, device="cuda"))
    keys = float32_keys(cache)
    for s in range(256):
        p = int(cache.table[s, 0, 0])
        codes, scale = summary_of(keys[p], 1)
        assert (summary.codes[p].cpu().numpy() == codes).all() and float(summary.scale[p]) == float(scale)
