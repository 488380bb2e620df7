"""Pools of pages as the library is told of them."""
import pytest
import torch

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
