"""4-bit pages without a GPU: the rule of the tests' own form, and what the C entry points refuse."""
import ctypes as C

import pytest
import torch

import four_bit as F
from paper_2502_03805_b200 import binding as B
from paper_2502_03805_b200 import build


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return B.load()


def _cache(**kw):
    base = dict(nseq=2, Hq=8, Hkv=2, dh=64, dtype="bf16", format="e2m1", page_size=32, num_pages=10, max_pages=4, k_pages=256,
                v_pages=512, page_table=64, k_scale=128, v_scale=192, k_group_scale=1024, v_group_scale=2048)
    return B.make_cache(**{**base, **kw})


@pytest.mark.parametrize("kw,status", [
    (dict(k_group_scale=None), B.CKV_EINVAL), (dict(v_group_scale=None), B.CKV_EINVAL), (dict(v_group_scale=1032), B.CKV_EALIGN),
    (dict(k_scale=None), B.CKV_EINVAL), (dict(k_pages=264), B.CKV_EALIGN), (dict(page_stride=32 * 64 - 32), B.CKV_EINVAL),
    (dict(page_stride=32 * 64 + 16), B.CKV_EALIGN), (dict(page_stride=32 * 64 + 31), B.CKV_EALIGN), (dict(format=4), B.CKV_EINVAL)])
def test_bad_descriptions_are_refused(lib, kw, status):
    fake, c, n = C.addressof(C.create_string_buffer(4096)), _cache(**kw), C.c_size_t()
    assert lib.criticalkv_decode_workspace_bytes(C.byref(c), C.byref(n)) == status
    assert B.criticalkv_decode(fake, c, 16, None, 16, 16, None, 256, ws_bytes=1 << 30, check=False) == status
    assert B.criticalkv_cache_store(fake, c, 16, 16, 1, None, None, None, 0, None, 16, 32, check=False) == status
    assert B.criticalkv_cache_load(fake, c, 16, 1, None, 0, 16, 16, check=False) == status


def test_a_good_description_is_taken_and_the_others_do_not_look_at_group_scales(lib):
    assert B.criticalkv_decode_workspace_bytes(_cache()) == B.criticalkv_decode_workspace_bytes(_cache(page_stride=32 * 64 + 32))
    assert B.criticalkv_decode_workspace_bytes(_cache(format="e4m3", k_group_scale=None, v_group_scale=3)) > 0


def test_codes_and_scales_of_the_plain_form():
    x = torch.tensor([0.0, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 2.51, 3.5, 5.0, 5.01, 9.0, -0.25, -0.75, -9.0, -0.0])
    assert F.encode(x.numpy()).tolist() == [0, 0, 1, 2, 2, 4, 4, 5, 6, 6, 7, 7, 8, 10, 15, 8]
    code, group, scale = F.quantise(x.repeat(4))
    assert code.shape == (32,) and group.shape == (4,) and float(scale) == float(torch.tensor(9.0) / 2688.0)
    # 9 / scale = 2688 = 448 * 6: the group with the largest element has the largest scale
    assert group.float().tolist() == [448.0] * 4
    g = torch.Generator().manual_seed(0)
    rows = torch.randn(200, 128, generator=g)
    back = F.values(*F.quantise(rows)).view(200, 8, 16)
    top = rows.view(200, 8, 16).abs().amax(-1, keepdim=True)
    # half the widest gap between codes (4 to 6) times a scale that is up to 1/16 off, and what is beyond 6 then
    assert bool(((back - rows.view(200, 8, 16)).abs() <= top / 6 * (1 + 2.0 ** -4) * 1.001).all())
