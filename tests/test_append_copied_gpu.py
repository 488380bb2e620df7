"""Elements that a rotation copies keep their bits in append as in rope and store, NaN with their payloads among them."""
import pytest
import torch

import cache_ref as R
from paper_2502_03805_b200 import PagedCache, Rotary, rope_frequencies
from test_append_gpu import make
from test_cache_gpu import gen, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dh,rot", [(128, 20), (128, 36), (64, 2), (64, 62), (128, 126), (128, 16), (64, 48), (128, 128)])
def test_bits(dtype, layout, dh, rot):
    Hq, Hkv, T = 3, 2, 37
    bits = torch.int16 if dtype == "bf16" else torch.int32
    nan = [0x7fc0, -0x40, 0x7f81, -0x7f] if dtype == "bf16" else [0x7fc00000, -0x400000, 0x7f800001, -0x7fffff]    # quiet and signalling
    rows = []
    for h in (Hq, Hkv, Hkv):
        x = torch.randn(1, h, T, dh, generator=gen(h)).to(R.DT[dtype])
        for e in range(rot, dh):                    # of the copied elements, every third
            if (e - rot) % 3 == 0:
                x.view(bits)[:, :, e % T::4, e] = nan[e % 4]
        rows.append(x.cuda())
    q, k, v = rows
    pos, start = torch.arange(T, dtype=torch.int32, device="cuda")[None], torch.full((1, Hkv), 3, dtype=torch.int32, device="cuda")
    rotary = Rotary(dh=dh, frequencies=rope_frequencies(rot), layout=layout, device="cuda:0")
    one, two = (PagedCache.allocate(nseq=1, Hq=Hq * Hkv, Hkv=Hkv, dh=dh, dtype=dtype, rows=50, page_size=16) for _ in range(2))
    q = q.repeat_interleave(Hkv, dim=1).contiguous()
    got, _ = one.append(q, k, v, pos, rotary, start)
    want, turned = rotary.rotate(q, k, pos)
    two.store(turned, v, start)
    copied = want.view(bits)[..., rot:]
    assert torch.equal(copied, q.view(bits)[..., rot:])
    assert torch.equal(got.view(bits), want.view(bits))
    assert torch.equal(one.k_pages.view(bits), two.k_pages.view(bits)) and torch.equal(one.v_pages.view(bits), two.v_pages.view(bits))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["plain", "e4m3", "int8", "e2m1"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dh,rot", [(128, 128), (128, 32), (64, 20), (64, 8), (128, 124)])
def test_rows_of_special_values(dtype, fmt, layout, dh, rot):
    """Infinities, NaN, the largest and smallest numbers and zeros at every place of a row, turned or copied: the bits of rope and store."""
    H, n = 2, dh + 6
    kw = dict(nseq=1, Hq=H, Hkv=H, dh=dh, dtype=dtype, page=16, cols=-(-n // 16))
    one, two = make(fmt, **kw), make(fmt, **kw)
    top, tiny = float(torch.finfo(R.DT[dtype]).max), float(torch.finfo(R.DT[dtype]).smallest_normal)
    special = torch.tensor([float("inf"), float("nan"), -top, tiny / 4, -float("inf"), -0.0, top, -float("nan"), tiny])
    rows = [torch.randn(1, H, n, dh, generator=gen(i)).to(R.DT[dtype]) for i in range(3)]
    for i, x in enumerate(rows):
        for e in range(dh):
            x[:, :, e, e] = special[(e + i) % len(special)].to(x.dtype)
            if e % 5 == 0:
                x[:, :, e, (e + rot // 2) % dh] = special[(e + 3) % len(special)].to(x.dtype)
        for j, value in enumerate((0.0, top, -top, tiny, tiny / 4)):
            x[:, :, dh + j] = value
    q, k, v = (x.cuda() for x in rows)
    pos, start = torch.arange(n, dtype=torch.int32, device="cuda")[None] * 7, torch.zeros(1, H, dtype=torch.int32, device="cuda")
    rotary = Rotary(dh=dh, frequencies=rope_frequencies(rot), layout=layout, device="cuda:0")
    got, _ = one.c.append(q, k, v, pos, rotary, start)
    want, turned = rotary.rotate(q, k, pos)
    two.c.store(turned, v, start)
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(got.view(bits), want.view(bits)) and same(one.bits(), two.bits())
    assert one.intact() and one.c.device_status() == 0
