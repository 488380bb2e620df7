"""A PagedCache whose library is a stand-in, without a GPU."""
import threading

import torch

from paper_2502_03805_b200 import PagedCache
from paper_2502_03805_b200 import binding as B
from paper_2502_03805_b200 import cache as cache_module


def cache(monkeypatch):
    """2 sequences of 2 KV heads, 4 query heads of 64, tables of 8 pages; `told`: the numbers of rows and pages of its calls."""
    monkeypatch.setattr(cache_module, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(cache_module, "_current_device", lambda: 0)
    monkeypatch.setattr(cache_module, "_capturing", lambda: False)
    told = []
    c = PagedCache.__new__(PagedCache)
    c.nseq, c.Hq, c.Hkv, c.dh, c.num_pages, c.max_pages = 2, 4, 2, 64, 9, 8
    c.dtype, c.torch_dtype, c.device, c._index = "bf16", torch.bfloat16, torch.device("cpu"), 0
    c.desc = B.make_cache(nseq=2, Hq=4, Hkv=2, dh=64, dtype="bf16", format="plain", page_size=16, num_pages=9, max_pages=8,
                          k_pages=256, v_pages=256, page_table=256)
    c.handle, c._owned, c._ref, c._plans, c._seen = None, False, None, {}, {0}
    c._ws, c._ws_bytes, c._parts, c._chosen, c._out_shape = {}, 256, {}, {}, (2, 4, 64)
    c._out_like, c._lse_like = torch.empty(2, 4, 64, dtype=torch.bfloat16), torch.empty(2, 4)
    c._load = lambda handle, ref, lens, n, strides, how, K, V, raw: told.append(n) or 0
    c._select = lambda handle, ref, q, strides, lens, codes, scale, pages, *rest: told.append(pages) or 0
    c._decode = lambda *args: 0
    c.told, c._lock = told, threading.Lock()
    return c
