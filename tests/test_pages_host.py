"""What appending, summaries and the choice of pages refuse before any CUDA call, without a GPU."""
import ctypes as C

import pytest

from paper_2502_03805_b200 import binding as B
from paper_2502_03805_b200 import build


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build_library()
    return B.load()


FAKE = C.create_string_buffer(4096)
HANDLE = C.addressof(FAKE)


def cache(**kw):
    base = dict(nseq=2, Hq=8, Hkv=2, dh=64, dtype="bf16", format="e4m3", page_size=32, num_pages=10, max_pages=4, k_pages=1 << 20,
                v_pages=1 << 21, page_table=1 << 16, k_scale=1 << 22, v_scale=1 << 23)
    return B.make_cache(**{**base, **kw})


def append(c=None, handle=HANDLE, v_stride=None, q=256, k=256, v=256, pos=1 << 14, freq=1 << 15, counts=None, start=4096, q_out=256,
           lens_out=None, reserved=0, **kw):
    r = B.make_rope_desc(**{**dict(nseq=2, T=3, Hq=8, Hk=2, dh=64, rot=64, dtype="bf16", layout="half"), **kw})
    r.reserved = reserved
    return B.criticalkv_cache_append(handle, c or cache(), r, q, k, v, v_stride, pos, freq, counts, start, q_out, lens_out, check=False)


def test_append():
    assert append(handle=None) == B.CKV_EINVAL and append(cache(dh=96)) == B.CKV_ENOTSUP
    for kw in (dict(nseq=1), dict(T=-1), dict(Hq=4), dict(Hk=1), dict(dh=128), dict(dtype="f32"), dict(rot=0), dict(rot=7), dict(rot=66),
               dict(layout=2), dict(factor=float("inf")), dict(reserved=1), dict(k_out_stride=(0, 0, 64)), dict(q=None), dict(k=None),
               dict(v=None), dict(pos=None), dict(freq=None), dict(q_out=None), dict(start=None), dict(q_stride=(0, 0, 32)),
               dict(v_stride=(0, -64, 0))):
        assert append(**kw) == B.CKV_EINVAL, kw
    for kw in (dict(q=264), dict(k=8), dict(v=24), dict(q_out=4), dict(pos=2), dict(freq=4), dict(counts=3), dict(start=1),
               dict(lens_out=4097), dict(k_stride=(0, 0, 68)), dict(v_stride=(0, 0, 68)), dict(q_out_stride=(4, 0, 0))):
        assert append(**kw) == B.CKV_EALIGN, kw
    for at in (4100, 4092, (1 << 14) + 20, (1 << 15) + 8, (1 << 16) + 4):          # start, positions, frequencies, page table
        assert append(lens_out=at) == B.CKV_EINVAL
    assert append(counts=8192, lens_out=8196) == B.CKV_EINVAL
    assert append(nseq=2, T=2 ** 30) == B.CKV_ENOTSUP
    assert append(cache(nseq=0), nseq=0) == B.CKV_OK


def summarise(c=None, handle=HANDLE, start=None, lens=4096, codes=256, scales=512):
    return B.criticalkv_summarise_pages(handle, c or cache(), start, lens, codes, scales, check=False)


def test_summarise():
    assert summarise(handle=None) == B.CKV_EINVAL and summarise(cache(page_size=8)) == B.CKV_ENOTSUP
    assert summarise(lens=None) == summarise(codes=None) == summarise(scales=None) == B.CKV_EINVAL
    assert summarise(lens=2) == summarise(codes=264) == summarise(scales=6) == summarise(start=1) == B.CKV_EALIGN
    assert summarise(cache(nseq=0), lens=None, codes=None, scales=None) == B.CKV_OK


def select(c=None, handle=HANDLE, q=256, q_stride=None, lens=4096, codes=256, scales=512, count=3, first=1, last=1, table=8192,
           rows=12288, chosen=None):
    return B.criticalkv_select_pages(handle, c or cache(), q, q_stride, lens, codes, scales, count, first, last, table, rows, chosen,
                                     check=False)


def test_select():
    assert select(handle=None) == B.CKV_EINVAL and select(cache(dtype=2)) == B.CKV_EINVAL
    for kw in (dict(count=0), dict(first=-1), dict(last=-1), dict(first=4), dict(first=2, last=2), dict(first=2 ** 31 - 1, last=2 ** 31 - 1),
               dict(q=None), dict(lens=None), dict(codes=None), dict(scales=None), dict(table=None), dict(rows=None), dict(q_stride=(-512, 0))):
        assert select(**kw) == B.CKV_EINVAL, kw
    for kw in (dict(q=264), dict(lens=2), dict(codes=8), dict(scales=2), dict(table=2), dict(rows=3), dict(chosen=1), dict(q_stride=(0, 68))):
        assert select(**kw) == B.CKV_EALIGN, kw
    # outputs over what is read, or over each other (2 x 2 heads of 3 pages: 48 bytes; lengths: 16)
    for kw in (dict(table=(1 << 16) + 60), dict(table=4096 - 44), dict(rows=4096 + 12), dict(rows=(1 << 16) - 12), dict(rows=8192 + 44),
               dict(chosen=8192 + 44), dict(chosen=12288 - 44), dict(chosen=4096 - 44), dict(chosen=(1 << 16) + 60)):
        assert select(**kw) == B.CKV_EINVAL, kw
    assert select(cache(max_pages=32769)) == select(cache(Hq=258)) == select(count=2 ** 26) == B.CKV_ENOTSUP
    assert select(cache(nseq=2 ** 25 + 1, Hq=2)) == B.CKV_ENOTSUP
    assert select(cache(nseq=0), q=None, lens=None, codes=None, scales=None, table=None, rows=None) == B.CKV_OK


def test_load_flags():
    load = lambda right: B.load().criticalkv_cache_load(HANDLE, C.byref(cache()), None, 4, None, right, 256, 256, None)  # noqa: E731
    assert B.CKV_LOAD_CLEAR == 256
    for right in (2, 3, 255, 258, 512, -1):
        assert load(right) == B.CKV_EINVAL
