"""Host-side checks of rotary positions, the paged cache and decode attention that need no GPU: what the C entry points
refuse before any CUDA call, and the frequency tables."""
import ctypes as C
import math

import pytest
import torch

from paper_2502_03805_b200 import binding as B
from paper_2502_03805_b200 import build, rope_frequencies
from paper_2502_03805_b200.cache import _row_strides


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return B.load()


@pytest.fixture(scope="module")
def fake():
    """A block of host memory standing in for a handle: calls that are refused never look at it."""
    return C.addressof(C.create_string_buffer(4096))


def _cache(**kw):
    base = dict(nseq=2, Hq=8, Hkv=2, dh=64, dtype="bf16", format="e4m3", page_size=32, num_pages=10, max_pages=4,
                k_pages=256, v_pages=512, page_table=64, k_scale=128, v_scale=192)
    base.update(kw)
    return B.make_cache(**base)


BAD_CACHES = [
    (dict(nseq=-1), B.CKV_EINVAL), (dict(Hq=7), B.CKV_EINVAL), (dict(Hkv=0), B.CKV_EINVAL),
    (dict(Hq=65, Hkv=65), B.CKV_ENOTSUP), (dict(Hq=1 << 17, Hkv=1), B.CKV_ENOTSUP), (dict(dh=96), B.CKV_ENOTSUP),
    (dict(dtype=2), B.CKV_EINVAL), (dict(format=3), B.CKV_EINVAL), (dict(format=-1), B.CKV_EINVAL),
    (dict(page_size=8), B.CKV_ENOTSUP), (dict(page_size=48), B.CKV_ENOTSUP), (dict(page_size=512), B.CKV_ENOTSUP),
    (dict(num_pages=0), B.CKV_EINVAL), (dict(max_pages=0), B.CKV_EINVAL), (dict(max_pages=1 << 27), B.CKV_ENOTSUP),
    (dict(flags=B.CKV_FLAG_WO_SHARED), B.CKV_EINVAL), (dict(scale=math.inf), B.CKV_EINVAL),
    (dict(scale=math.nan), B.CKV_EINVAL), (dict(page_stride=32 * 64 - 16), B.CKV_EINVAL),
    (dict(page_stride=32 * 64 + 8), B.CKV_EALIGN), (dict(k_pages=None), B.CKV_EINVAL), (dict(v_scale=None), B.CKV_EINVAL),
    (dict(k_pages=264), B.CKV_EALIGN), (dict(k_scale=132), B.CKV_EALIGN), (dict(page_table=66), B.CKV_EALIGN),
    (dict(page_table=None), B.CKV_EINVAL), (dict(nseq=1 << 30), B.CKV_ENOTSUP),
]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_bad_cache_descriptions_are_refused_by_every_call(lib, fake, kw, status):
    c = _cache(**kw)
    n = C.c_size_t()
    assert lib.criticalkv_decode_workspace_bytes(C.byref(c), C.byref(n)) == status
    assert B.criticalkv_decode(fake, c, 16, None, 16, 16, None, 256, ws_bytes=1 << 30, check=False) == status
    assert B.criticalkv_cache_store(fake, c, 16, 16, 1, None, None, None, 0, None, 16, 32, check=False) == status
    assert B.criticalkv_cache_load(fake, c, 16, 1, None, 0, 16, 16, check=False) == status


def test_reserved_fields_must_be_zero(lib, fake):
    c = _cache()
    c.reserved = 1
    assert B.criticalkv_cache_load(fake, c, 16, 1, None, 0, 16, 16, check=False) == B.CKV_EINVAL
    d = B.make_rope_desc(nseq=1, T=1, Hq=1, Hk=0, dh=64, rot=64, dtype="f32", layout="half")
    d.reserved = 1
    assert B.criticalkv_rope(fake, d, 16, None, 16, 16, 16, None, check=False) == B.CKV_EINVAL


def test_decode_workspace(lib):
    small, large = (B.criticalkv_decode_workspace_bytes(_cache(Hq=2 * g)) for g in (4, 32))
    assert small % 256 == 0 and large > small
    # the sizes depend neither on the number of sequences nor on the table
    assert B.criticalkv_decode_workspace_bytes(_cache(nseq=100, max_pages=1000)) == small


def test_decode_refuses_bad_arguments(lib, fake):
    c = _cache()
    ok = dict(q=256, q_stride=None, lens=256, out=256, lse=None, ws=256, ws_bytes=1 << 30)

    def rc(handle=fake, **kw):
        a = {**ok, **kw}
        return B.criticalkv_decode(handle, c, a["q"], a["q_stride"], a["lens"], a["out"], a["lse"], a["ws"],
                                   ws_bytes=a["ws_bytes"], check=False)
    assert rc(handle=None) == B.CKV_EINVAL
    for name in ("q", "lens", "out", "ws"):
        assert rc(**{name: None}) == B.CKV_EINVAL
    for name, at in (("q", 8), ("out", 24), ("lens", 2), ("lse", 6), ("ws", 128)):
        assert rc(**{name: at}) == B.CKV_EALIGN
    assert rc(q_stride=(0, 68)) == B.CKV_EALIGN and rc(q_stride=(-512, 0)) == B.CKV_EINVAL
    assert rc(ws_bytes=B.criticalkv_decode_workspace_bytes(c) - 1) == B.CKV_EWORKSPACE
    huge = _cache(nseq=1 << 12, max_pages=1 << 23)          # more tiles than 32 bits count
    assert B.criticalkv_decode(fake, huge, 256, None, 256, 256, None, 256, ws_bytes=1 << 30, check=False) == B.CKV_ENOTSUP
    assert B.criticalkv_decode(fake, _cache(nseq=0), None, None, None, None, None, None, ws_bytes=0, check=False) == B.CKV_OK


def test_store_and_load_refuse_bad_arguments(lib, fake):
    c = _cache()

    def store(K=256, V=256, n=4, stride=None, idx=None, offsets=None, idx_rows=0, counts=None, start=256, lens_out=None):
        return B.criticalkv_cache_store(fake, c, K, V, n, stride, idx, offsets, idx_rows, counts, start, lens_out,
                                        check=False)

    assert store(n=-1) == B.CKV_EINVAL and store(K=None) == B.CKV_EINVAL and store(start=None) == B.CKV_EINVAL
    assert store(idx=256) == B.CKV_EINVAL and store(offsets=256) == B.CKV_EINVAL
    assert store(idx=256, offsets=256, counts=256) == B.CKV_EINVAL and store(idx_rows=-1) == B.CKV_EINVAL
    assert store(idx=256, offsets=256, idx_rows=1 << 31) == B.CKV_ENOTSUP
    assert store(K=264) == B.CKV_EALIGN and store(start=258) == B.CKV_EALIGN and store(counts=2) == B.CKV_EALIGN
    assert store(stride=(0, 0, 68)) == B.CKV_EALIGN and store(stride=(0, 0, 32)) == B.CKV_EINVAL
    assert store(stride=(0, -64, 0)) == B.CKV_EINVAL
    assert store(start=256, lens_out=264) == B.CKV_EINVAL        # overlaps start without being it
    assert B.criticalkv_cache_store(None, c, 256, 256, 1, None, None, None, 0, None, 256, None, check=False) == B.CKV_EINVAL

    def load(lens=256, n=4, stride=None, right=0, K=256, V=256):
        return B.load().criticalkv_cache_load(fake, C.byref(c), lens, n, B._strides(stride), right, K, V, None)

    assert load(n=-1) == B.CKV_EINVAL and load(right=2) == B.CKV_EINVAL and load(lens=None) == B.CKV_EINVAL
    assert load(K=None) == B.CKV_EINVAL and load(V=260) == B.CKV_EALIGN and load(lens=255) == B.CKV_EALIGN
    assert load(n=0, lens=None, K=None, V=None) == B.CKV_OK
    assert load(stride=(0, 0, 60)) == B.CKV_EALIGN


@pytest.mark.parametrize("kw,status", [
    (dict(nseq=-1), B.CKV_EINVAL), (dict(T=-1), B.CKV_EINVAL), (dict(Hq=0), B.CKV_EINVAL), (dict(Hk=-1), B.CKV_EINVAL),
    (dict(Hq=5000), B.CKV_ENOTSUP), (dict(dh=60), B.CKV_EINVAL), (dict(dh=264, rot=64), B.CKV_ENOTSUP),
    (dict(rot=0), B.CKV_EINVAL), (dict(rot=7), B.CKV_EINVAL), (dict(rot=66), B.CKV_EINVAL), (dict(dtype=5), B.CKV_EINVAL),
    (dict(layout=2), B.CKV_EINVAL), (dict(factor=math.nan), B.CKV_EINVAL), (dict(factor=math.inf), B.CKV_EINVAL),
    (dict(q_stride=(0, 0, 68)), B.CKV_EALIGN), (dict(q_stride=(0, 0, 56)), B.CKV_EINVAL),
    (dict(k_out_stride=(0, -64, 0)), B.CKV_EINVAL), (dict(nseq=1 << 16, T=1 << 16), B.CKV_ENOTSUP),
])
def test_bad_rope_descriptions_are_refused(lib, fake, kw, status):
    base = dict(nseq=1, T=4, Hq=2, Hk=1, dh=64, rot=64, dtype="bf16", layout="half")
    d = B.make_rope_desc(**{**base, **kw})
    assert B.criticalkv_rope(fake, d, 16, 16, 16, 16, 16, 16, check=False) == status


def test_rope_refuses_bad_pointers_and_ignores_empty_calls(lib, fake):
    d = B.make_rope_desc(nseq=1, T=4, Hq=2, Hk=1, dh=64, rot=64, dtype="bf16", layout="half")
    good = [16] * 6
    for i, at, want in [(0, None, B.CKV_EINVAL), (1, None, B.CKV_EINVAL), (2, None, B.CKV_EINVAL), (3, None, B.CKV_EINVAL),
                        (5, None, B.CKV_EINVAL), (0, 8, B.CKV_EALIGN), (2, 2, B.CKV_EALIGN), (3, 4, B.CKV_EALIGN),
                        (5, 24, B.CKV_EALIGN)]:
        a = list(good)
        a[i] = at
        assert B.criticalkv_rope(fake, d, *a, check=False) == want
    assert B.criticalkv_rope(None, d, *good, check=False) == B.CKV_EINVAL
    for kw in (dict(nseq=0, T=4), dict(nseq=1, T=0)):
        e = B.make_rope_desc(Hq=2, Hk=1, dh=64, rot=64, dtype="bf16", layout="half", **kw)
        assert B.criticalkv_rope(fake, e, *[None] * 6, check=False) == B.CKV_OK


def test_strides_handed_to_the_library():
    x = torch.zeros(2, 5, 6, 64)
    assert _row_strides(x, "x") is None
    assert _row_strides(x.transpose(1, 2), "x") == (5 * 6 * 64, 64, 6 * 64)
    assert _row_strides(x[:, :, ::2], "x") == (5 * 6 * 64, 6 * 64, 128)
    assert _row_strides(x[:, 1:2, ::2], "x") == (5 * 6 * 64, 3 * 64, 128)   # the stride of a single head is not used
    with pytest.raises(ValueError):
        _row_strides(x[:, :1].expand(2, 5, 6, 64), "x")                     # repeated heads
    with pytest.raises(ValueError):
        _row_strides(x[..., ::2], "x")


# ---- frequencies: against formulas written out once more -----------------------------------------------------------
def test_plain_frequencies():
    f = rope_frequencies(8, 10000.0)
    assert f.dtype == torch.float64
    assert f.tolist() == pytest.approx([1.0, 0.1, 0.01, 0.001], rel=1e-14)
    assert rope_frequencies(8, 10000.0, "linear", factor=4.0).tolist() == pytest.approx([0.25, 0.025, 0.0025, 0.00025], rel=1e-14)


def test_ntk_keeps_the_fastest_pair_and_divides_the_slowest():
    a, b = rope_frequencies(64, 10000.0), rope_frequencies(64, 10000.0, "ntk", factor=8.0)
    assert b[0].item() == a[0].item() == 1.0
    assert (a[-1] / b[-1]).item() == pytest.approx(8.0, rel=1e-12)


def test_llama3_bands():
    a = rope_frequencies(128, 500000.0)
    b = rope_frequencies(128, 500000.0, "llama3", factor=8.0, original=8192, low=1.0, high=4.0)
    for x, y in zip(a.tolist(), b.tolist()):
        wave = 2 * math.pi / x
        if wave < 8192 / 4:
            want = x
        elif wave > 8192:
            want = x / 8
        else:
            t = (8192 / wave - 1) / 3
            want = (1 - t) * x / 8 + t * x
        assert y == pytest.approx(want, rel=1e-13)


def test_yarn_ramp():
    a = rope_frequencies(128, 10000.0)
    b = rope_frequencies(128, 10000.0, "yarn", factor=16.0, original=4096)
    r = (b / a).tolist()
    lo = max(math.floor(128 * math.log(4096 / (32 * 2 * math.pi)) / (2 * math.log(10000))), 0)
    hi = math.ceil(128 * math.log(4096 / (2 * math.pi)) / (2 * math.log(10000)))
    for i, x in enumerate(r):
        t = min(max((i - lo) / (hi - lo), 0.0), 1.0)
        assert x == pytest.approx((1 - t) + t / 16, rel=1e-12)


@pytest.mark.parametrize("kw", [dict(rot=7), dict(rot=0), dict(rot=8, scaling="other"), dict(rot=8, scaling="linear", factor=0.5),
                                dict(rot=2, scaling="ntk", factor=2.0), dict(rot=8, scaling="llama3", low=4.0, high=1.0),
                                dict(rot=8, scaling="yarn", beta_fast=1.0, beta_slow=2.0), dict(rot=8, base=1.0)])
def test_bad_frequency_arguments(kw):
    with pytest.raises(ValueError):
        rope_frequencies(**kw)
