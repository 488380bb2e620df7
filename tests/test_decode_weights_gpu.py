"""How many bits the weights of decode attention have: heads in which the values cancel, and heads in which many rows of
little weight stand beside one that has nearly all of it."""
import math

import pytest
import torch

import cache_ref as R
import decode_bounds as D
from paper_2502_03805_b200 import PagedCache
from paper_2502_03805_b200 import binding as B

pytestmark = pytest.mark.gpu


def attend(dtype, fmt, kernel, k, ks, v, vs, q, scale, page=16):
    """One KV head of the rows k, v [n, dh] (codes with the row scales ks, vs, or plain rows): got, want, lens."""
    n, dh = k.shape
    cols = -(-n // page)
    code = R.CODE.get(fmt, R.DT[dtype])
    pages = [torch.zeros(cols * page, dh) for _ in range(2)]
    scales = [torch.ones(cols * page) for _ in range(2)]
    for p, s, x, xs in ((pages[0], scales[0], k, ks), (pages[1], scales[1], v, vs)):
        p[:n] = x if fmt != "plain" else x * xs[:, None]
        s[:n] = xs
    pages = [p.to(code).view(cols, page, dh) for p in pages]
    scales = [s.view(cols, page) for s in scales]
    table = torch.arange(cols, dtype=torch.int32).view(1, 1, cols)
    dev = [x.cuda() for x in pages + scales]
    c = PagedCache(Hq=q.shape[1], dtype=dtype, format=fmt, k_pages=dev[0], v_pages=dev[1], page_table=table.cuda(),
                   k_scale=dev[2] if fmt != "plain" else None, v_scale=dev[3] if fmt != "plain" else None, scale=scale,
                   flags=B.CKV_FLAG_FORCE_SIMT if kernel == "cuda" else 0)
    lens = torch.full((1, 1), n, dtype=torch.int32)
    q_dev, lens_dev = q.cuda(), lens.cuda()
    torch.cuda.synchronize()
    got = c.attend(q_dev, lens_dev)
    torch.cuda.synchronize()
    assert B.criticalkv_last_path(c.handle) & 384 == (128 if kernel == "tensor" else 256)
    kv, vv = (R.stored(p, s, fmt) for p, s in ((pages[0], scales[0]), (pages[1], scales[1])))
    want = D.decode(q, kv, vv, table, lens, page, scale, fmt, dtype, kernel, scales[1])
    return got, want, lens


PATHS = [("bf16", "e4m3", "tensor"), ("bf16", "int8", "tensor"), ("bf16", "plain", "tensor"), ("bf16", "e4m3", "cuda"),
         ("bf16", "plain", "cuda"), ("f32", "e4m3", "cuda"), ("f32", "int8", "cuda"), ("f32", "plain", "cuda")]


@pytest.mark.parametrize("dtype,fmt,kernel", PATHS)
@pytest.mark.parametrize("dh,G", [(64, 1), (128, 4), (64, 8), (128, 16)])
@pytest.mark.parametrize("pairs", [1, 9, 150])
def test_values_that_cancel(dtype, fmt, kernel, dh, G, pairs):
    """Pairs of rows with opposite values whose weights differ by less than 2^-9: what is left is that difference, which a
    weight of 11 bits has nothing of."""
    n = 2 * pairs
    k = torch.zeros(n, dh)
    k[:, 0] = 1.0
    ks = torch.ones(n)
    if fmt == "plain" and dtype == "bf16":
        k[1::2, 0], k[:, 1] = 1.0 - 2.0 ** -8, 2.0 ** -4                        # bf16 rows cannot be closer
    else:
        ks[1::2] = 1.0 - 2.0 ** -12 * torch.arange(1, pairs + 1).remainder(5).add(1).float()
    v = torch.ones(n, dh)
    v[1::2] = -1.0
    v[:, 1::2] *= -1.0
    q = torch.zeros(1, G, dh)
    q[..., 0] = 1.0 + torch.arange(G).float() / 16
    got, want, lens = attend(dtype, fmt, kernel, k, ks, v, torch.ones(n), q.to(R.DT[dtype]), 0.25)
    assert float(want[0].abs().max()) < 2.0 ** -9 and float((want[2] / want[0].abs()).max()) < 0.3   # the bound is narrow
    D.check(got, want, lens, G)


@pytest.mark.parametrize("dtype,fmt,kernel", PATHS)
@pytest.mark.parametrize("dh,G", [(64, 1), (128, 4), (64, 8), (128, 16)])
@pytest.mark.parametrize("n", [100, 3001])
@pytest.mark.parametrize("octaves", [18.0, 25.75, 33.0])
def test_a_long_tail_beside_one_strong_row(dtype, fmt, kernel, dh, G, n, octaves):
    """One row has nearly all the weight and zeros in the odd elements; the others are 2^-octaves as heavy and have the odd
    elements to themselves."""
    at = n // 3
    k = torch.zeros(n, dh)
    k[:, 0] = -1.0
    k[at, 0] = 1.0
    v = torch.ones(n, dh)
    v[at, 1::2] = 0.0
    q = torch.zeros(1, G, dh)
    q[..., 0] = 1.0
    got, want, lens = attend(dtype, fmt, kernel, k, torch.ones(n), v, torch.ones(n), q.to(R.DT[dtype]),
                             octaves * math.log(2.0) / 2)
    tail = want[0][..., 1::2]
    assert bool((tail > 0.9 * (n - 1) * 2.0 ** -octaves / (1 + (n - 1) * 2.0 ** -octaves)).all())
    assert float((want[2][..., 1::2] / tail).max()) < 0.05
    D.check(got, want, lens, G)
