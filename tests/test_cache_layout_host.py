"""Pools of pages as the library is told of them."""
import ctypes as C

import pytest
import torch

from paper_2502_03805_b200 import binding as B
from paper_2502_03805_b200 import build
from paper_2502_03805_b200 import cache as cache_module


def test_page_strides():
    x = torch.zeros(5, 16, 64)
    assert cache_module._page_stride(x, "x") == 16 * 64
    assert cache_module._page_stride(torch.zeros(5, 2, 16, 64)[:, 1], "x") == 2 * 16 * 64
    assert cache_module._page_stride(x[:1], "x") == cache_module._page_stride(x[:1].expand(1, 16, 64), "x") == 16 * 64
    for bad in (x[:1].expand(5, 16, 64),                                  # one page five times: stride 0 would mean dense
                x.flatten().as_strided((5, 16, 64), (8 * 64, 64, 1)),     # every page over half of the next
                torch.zeros(5, 16, 128)[..., :64], torch.zeros(5, 32, 64)[:, ::2], torch.zeros(5, 64, 16).transpose(1, 2)):
        with pytest.raises(ValueError):
            cache_module._page_stride(bad, "x")


def test_lengths_may_not_overlap_what_a_store_reads():
    """Every CTA of a head reads the counts, offsets and indices, one writes the new length: only `start` is read in a way
    that allows it to be that array."""
    build.build_library()
    B.load()
    fake = C.addressof(C.create_string_buffer(4096))
    c = B.make_cache(nseq=2, Hq=2, Hkv=1, dh=64, dtype="bf16", format="plain", page_size=16, num_pages=4, max_pages=3,
                     k_pages=1 << 20, v_pages=1 << 21, page_table=1 << 16)

    def store(lens_out, counts=None, idx=None, offsets=None, start=4096):
        return B.criticalkv_cache_store(fake, c, 1 << 22, 1 << 23, 8, None, idx, offsets, 5 if idx else 0, counts, start,
                                        lens_out, check=False)

    for at in (8192, 8196):
        assert store(at, counts=8192) == store(8192, counts=at) == B.CKV_EINVAL
    assert store(8192, idx=12288, offsets=8192) == store(8192 + 12, idx=12288, offsets=8192) == B.CKV_EINVAL
    assert store(12288 + 36, idx=12288, offsets=8192) == B.CKV_EINVAL
    assert store((1 << 16) + 20) == store((1 << 16) - 4) == B.CKV_EINVAL
    assert store(4096 + 4) == store(4096 - 4) == B.CKV_EINVAL


def test_counts_that_pass_32_bits_inside_a_kernel_are_refused():
    build.build_library()
    B.load()
    fake = C.addressof(C.create_string_buffer(4096))

    def rope(nseq, T):       # the last tile of tokens may reach 255 tokens behind T
        d = B.make_rope_desc(nseq=nseq, T=T, Hq=1, Hk=0, dh=8, rot=2, dtype="f32", layout="half")
        return B.criticalkv_rope(fake, d, 16, None, 16, None, 16, None, check=False)      # refused for the null otherwise

    assert rope(1, 2 ** 31 - 256) == rope(1, 2 ** 31 - 1) == rope(3, 2 ** 30) == B.CKV_ENOTSUP
    assert rope(1, 2 ** 31 - 257) == rope(2, 2 ** 29) == B.CKV_EINVAL

    def decode(nseq, Hq, Hkv):
        c = B.make_cache(nseq=nseq, Hq=Hq, Hkv=Hkv, dh=64, dtype="bf16", format="plain", page_size=16, num_pages=4, max_pages=1,
                         k_pages=1 << 20, v_pages=1 << 21, page_table=1 << 16)
        return B.criticalkv_decode(fake, c, None, None, 256, 256, None, 256, ws_bytes=1 << 30, check=False)

    assert decode((1 << 23) + 1, 8, 8) == decode(1 << 25, 24, 1) == B.CKV_ENOTSUP
    assert decode(1 << 23, 8, 8) == decode(1 << 25, 16, 1) == B.CKV_EINVAL
