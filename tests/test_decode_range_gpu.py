"""8-bit pages whose row scales are far from 1, with queries that make up for it: the logits are ordinary numbers."""
import pytest
import torch

import cache_ref as R
import decode_bounds as D
from test_cache_gpu import Cache, gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("exponent", [-80, -40, 40, 80, 110])
def test_rows_far_from_one(dtype, fmt, exponent):
    """Keys 2^exponent large under queries of 2^-exponent; values of 2^-exponent."""
    lens = torch.tensor([[70, 33]], dtype=torch.int32)
    cache = Cache(nseq=1, Hq=8, Hkv=2, dh=64, dtype=dtype, fmt=fmt, page=16, cols=5).fill(lens, 3, spread=0.3)
    cache.ks.mul_(2.0 ** exponent)
    cache.vs.mul_(2.0 ** -exponent)
    q = (torch.randn(1, 8, 64, generator=gen(8)) * 2.0 ** -exponent).to(R.DT[dtype])
    q_dev, lens_dev = q.cuda(), lens.cuda()
    torch.cuda.synchronize()
    got = cache.c.attend(q_dev, lens_dev)
    kv, vv = cache.values()
    D.check(got, D.decode(q, kv, vv, cache.table, lens, 16, 0.125, fmt, dtype, "tensor" if dtype == "bf16" else "cuda", cache.vs,
                          16), lens, 4)
