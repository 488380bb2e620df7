"""Decoding on a compressed cache: rotary positions, the paged cache, and attention of a new token over it.

Device-buffer plumbing around the C ABI, like session.py: shapes, types and devices of tensors are checked here, every
number is computed by the kernels of libcriticalkv.  Work goes to torch's current stream of the tensors' device unless
a stream is given.  The tensors of a call must be ready on that stream; what an object keeps for itself (pages, tables,
frequencies, workspaces) may be dropped while calls are in flight on torch's own streams.  On a stream that torch did not
make (an address, torch.cuda.ExternalStream) the caller keeps the object until the calls are done.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import math

import torch

from . import binding as B

_TORCH_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_NAME = {v: k for k, v in _TORCH_DTYPE.items()}
_NOTHING = contextlib.nullcontext()
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (     # handle of a device's current stream
    lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_capturing = torch.cuda.is_current_stream_capturing
_CODE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def _sig(t):
    """What the checks of a tensor look at (None for an absent one)."""
    return None if t is None else (t.dtype, t.shape, t.stride(), t.get_device())


class _Owner:
    """The handle of an object: the caller's, or one of its own that is destroyed with it.

    A decode step is a handful of microseconds, so a call whose tensors have the types, shapes, strides and devices of
    an earlier one does not repeat the checks: `_plans` keeps what they came to (strides and descriptors for the C ABI).
    The calls spell out the signatures of their tensors (a function call for each would cost as much as a launch)."""

    def _take_handle(self, handle, device):
        if getattr(handle, "device", device.index) != device.index:
            raise ValueError(f"the handle is of device {handle.device}, the tensors are on {device}")
        self._owned = handle is None
        self.handle = B.criticalkv_create(device.index) if handle is None else handle
        self._plans = {}
        self._seen = set()               # streams that the tensors the object keeps are recorded on
        self._lib = B.load()
        self._index = device.index

    def _keep(self, key, plan):
        if len(self._plans) >= 256:      # prompts of ever new lengths
            self._plans.clear()
        self._plans[key] = plan
        return plan

    def close(self):
        if getattr(self, "_owned", False) and self.handle is not None:
            B.criticalkv_destroy(self.handle)
        self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _on(self, stream):
        if stream is None:
            return _raw_stream(self._index)
        return stream if isinstance(stream, int) else stream.cuda_stream

    def _torch_stream(self, stream):
        if stream is None:
            return torch.cuda.current_stream(self.device)
        if isinstance(stream, int):
            return torch.cuda.ExternalStream(stream, device=self.device) if stream else \
                torch.cuda.default_stream(self.device)
        return stream

    def _allocating(self, stream):
        """Where outputs of a call on `stream` are allocated and cleared: on that stream, not on the current one."""
        return _NOTHING if stream is None else torch.cuda.stream(self._torch_stream(stream))

    def _where(self, stream):
        """The stream of a call for the C ABI.  On its first call there, the tensors that the object keeps are recorded on
        it: their memory is not handed out again before the work in flight on it at their end is done."""
        raw = _raw_stream(self._index) if stream is None else self._on(stream)
        if raw not in self._seen:
            self._record(self._kept(), stream)
            self._seen.add(raw)
        return raw

    def _record(self, tensors, stream):
        at = self._torch_stream(stream)
        if at.cuda_stream and at.stream_id == at.cuda_stream:
            return       # not torch's: it may be gone when the tensors go, and an event would then be recorded on it
        for t in tensors:
            if t is not None:
                t.record_stream(at)

    def _fail(self, rc, where):
        B._check(self.handle, rc, where, True)

    def device_status(self, stream=None):
        return B.criticalkv_device_status(self.handle, self._on(stream))


def _device_of(t, what):
    if not t.is_cuda:
        raise ValueError(f"{what} is not on a CUDA device")
    return t.device


def _need(t, what, shape, dtype, device, dense=True):
    if t.dtype != dtype or t.device != device or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: need {dtype} {tuple(shape)} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    if dense and not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t


def _row_strides(t, what):
    """Element strides of all but the last dimension for the C ABI (0 = dense): rows must be contiguous, and a
    dimension repeated with stride 0 cannot be expressed."""
    if t.is_contiguous():
        return None
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{what}: the elements of a row must be contiguous")
    out, dense = [], 1
    for size, step in zip(t.shape[::-1], t.stride()[::-1]):
        if size > 1 and step == 0:
            raise ValueError(f"{what}: a dimension expanded with stride 0 is not supported")
        out.append(step if size > 1 else dense)
        dense *= max(size, 1)
    return tuple(out[:0:-1])


def _page_stride(t, what):
    """Elements from page to page of a pool whose pages are contiguous and apart (the C ABI takes 0 for dense)."""
    _, page_size, dh = t.shape
    if t.is_contiguous():
        return page_size * dh
    if t.stride(2) != 1 or t.stride(1) != dh:
        raise ValueError(f"{what}: the rows of a page must be contiguous")
    if t.stride(0) < page_size * dh:
        raise ValueError(f"{what}: pages expanded or laid over each other are not supported")
    return t.stride(0)


def rope_frequencies(rot, base=10000.0, scaling=None, *, factor=1.0, original=8192, low=1.0, high=4.0, beta_fast=32.0,
                     beta_slow=1.0):
    """Radians per position of the rot/2 pairs, as a float64 CPU tensor: base^(-2i/rot), adjusted for long contexts.

    scaling None     as it is
    "linear"         every frequency divided by `factor` (positions interpolated)
    "ntk"            base raised to base * factor^(rot / (rot - 2)): the slowest pair divided by `factor`, the fastest kept
    "llama3"         wavelengths above original/low divided by `factor`, below original/high kept, blended between
    "yarn"           pairs turning fewer than beta_slow times over `original` positions divided by `factor`, more than
                     beta_fast times kept, a linear ramp over the pair index between (its attention factor,
                     0.1 ln(factor) + 1, is Rotary's `factor` argument)
    """
    if rot < 2 or rot % 2:
        raise ValueError("rot must be even and at least 2")
    if not (factor >= 1.0 and base > 1.0 and original > 0):
        raise ValueError("need factor >= 1, base > 1 and original > 0")
    i = torch.arange(rot // 2, dtype=torch.float64)
    if scaling == "ntk":
        if rot == 2:
            raise ValueError('"ntk" needs rot > 2')
        base = base * factor ** (rot / (rot - 2))
    freq = torch.pow(torch.tensor(float(base), dtype=torch.float64), -2.0 * i / rot)
    if scaling in (None, "ntk"):
        return freq
    if scaling == "linear":
        return freq / factor
    if scaling == "llama3":
        if not high > low > 0:
            raise ValueError("need high > low > 0")
        turns = original * freq / (2.0 * math.pi)
        keep = ((turns - low) / (high - low)).clamp(0.0, 1.0)
    elif scaling == "yarn":
        if not beta_fast > beta_slow > 0:
            raise ValueError("need beta_fast > beta_slow > 0")

        def pair(turns):   # the (real-valued) pair index that turns so often over `original` positions
            return rot * math.log(original / (turns * 2.0 * math.pi)) / (2.0 * math.log(base))

        lo = max(math.floor(pair(beta_fast)), 0)
        hi = min(math.ceil(pair(beta_slow)), rot - 1)
        keep = 1.0 - ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
    else:
        raise ValueError(f"unknown scaling {scaling!r}")
    return (1.0 - keep) * freq / factor + keep * freq


class Rotary(_Owner):
    """Rotary positions for heads of dh elements, of which the first 2 * len(frequencies) are turned.

    frequencies: radians per position of each pair (rope_frequencies, or any float64 tensor); layout "half" (pairs
    i, i + rot/2) or "interleaved" (2i, 2i + 1); factor multiplies the turned part."""

    def __init__(self, *, dh, frequencies, layout="half", factor=1.0, device=None, handle=None):
        if layout not in ("half", "interleaved"):
            raise ValueError(f"unknown layout {layout!r}")
        if frequencies.dtype != torch.float64 or frequencies.dim() != 1:
            raise ValueError("frequencies must be a float64 vector")
        self.freq = frequencies.contiguous() if frequencies.is_cuda and device is None else frequencies.to(
            torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)).contiguous()
        self.device = _device_of(self.freq, "frequencies")
        self.dh, self.rot, self.layout, self.factor = dh, 2 * self.freq.numel(), layout, float(factor)
        self._take_handle(handle, self.device)
        self._rope, self._freq_at = self._lib.criticalkv_rope, self.freq.data_ptr()

    def rotate(self, q, k, positions, q_out=None, k_out=None, stream=None):
        """q [nseq, Hq, T, dh] and k [nseq, Hk, T, dh] (or None), any strides with contiguous rows; positions int32
        [nseq, T].  Returns (q_out, k_out); the outputs may be the inputs themselves."""
        if q_out is None or (k_out is None and k is not None):
            with self._allocating(stream):
                q_out = torch.empty(q.shape, dtype=q.dtype, device=self.device) if q_out is None else q_out
                if k is not None and k_out is None:
                    k_out = torch.empty(k.shape, dtype=k.dtype, device=self.device)
        key = (q.dtype, q.shape, q.stride(), q.get_device(), _sig(k), positions.dtype, positions.shape, positions.stride(),
               positions.get_device(), q_out.dtype, q_out.shape, q_out.stride(), q_out.get_device(), _sig(k_out))
        desc = self._plans.get(key) or self._keep(key, self._describe(q, k, positions, q_out, k_out))
        rc = self._rope(self.handle, desc, q.data_ptr(), None if k is None else k.data_ptr(), positions.data_ptr(),
                        self._freq_at, q_out.data_ptr(), None if k is None else k_out.data_ptr(), self._where(stream))
        if rc:
            self._fail(rc, "criticalkv_rope")
        return q_out, k_out

    def _kept(self):
        return (self.freq,)

    def _describe(self, q, k, positions, q_out, k_out):
        """Checks the tensors of a call and describes them to the C ABI."""
        if q.dim() != 4 or q.shape[3] != self.dh or q.dtype not in _NAME:
            raise ValueError(f"q: need [nseq, Hq, T, {self.dh}] of float32 or bfloat16")
        nseq, Hq, T, dh = q.shape
        dev = self.device
        _need(q, "q", q.shape, q.dtype, dev, dense=False)
        _need(positions, "positions", (nseq, T), torch.int32, dev)
        _need(q_out, "q_out", q.shape, q.dtype, dev, dense=False)
        zero, Hk, ks, kos = (0, 0, 0), 0, None, None
        if k is not None:
            if k.dim() != 4:
                raise ValueError("k must be [nseq, Hk, T, dh]")
            Hk = k.shape[1]
            _need(k, "k", (nseq, Hk, T, dh), q.dtype, dev, dense=False)
            _need(k_out, "k_out", k.shape, q.dtype, dev, dense=False)
            ks, kos = _row_strides(k, "k"), _row_strides(k_out, "k_out")
        elif k_out is not None:
            raise ValueError("k_out without k")
        return B.make_rope_desc(nseq=nseq, T=T, Hq=Hq, Hk=Hk, dh=dh, rot=self.rot, dtype=_NAME[q.dtype],
                                layout=self.layout, factor=self.factor, q_stride=_row_strides(q, "q") or zero,
                                k_stride=ks or zero, q_out_stride=_row_strides(q_out, "q_out") or zero,
                                k_out_stride=kos or zero)


class PagedCache(_Owner):
    """A paged KV cache whose heads have lengths of their own.

    k_pages, v_pages [num_pages, page_size, dh] of the model's type ("plain") or of 8-bit codes ("e4m3": float8_e4m3fn,
    "int8": int8) with k_scale, v_scale float32 [num_pages, page_size]; page_table int32 [nseq, Hkv, max_pages].  The
    tensors stay the caller's: lengths are passed to every call, pages are handed out by whoever owns the pool
    (PagedCache.allocate makes a pool in which every head has all its pages)."""

    def __init__(self, *, Hq, dtype, k_pages, v_pages, page_table, format="plain", k_scale=None, v_scale=None, scale=0.0,
                 flags=0, handle=None):
        if dtype not in _TORCH_DTYPE or format not in ("plain", "e4m3", "int8"):
            raise ValueError(f"unknown dtype {dtype!r} or format {format!r}")
        if k_pages.dim() != 3 or page_table.dim() != 3:
            raise ValueError("k_pages must be [num_pages, page_size, dh], page_table [nseq, Hkv, max_pages]")
        self.dtype, self.format, self.torch_dtype = dtype, format, _TORCH_DTYPE[dtype]
        dev = self.device = _device_of(k_pages, "k_pages")
        num_pages, page_size, dh = k_pages.shape
        code = _CODE.get(format, self.torch_dtype)
        strides = []
        for t, what in ((k_pages, "k_pages"), (v_pages, "v_pages")):
            _need(t, what, k_pages.shape, code, dev, dense=False)
            strides.append(_page_stride(t, what))
        if strides[0] != strides[1]:
            raise ValueError("k_pages and v_pages must have the same page stride")
        if (k_scale is None) != (format == "plain") or (v_scale is None) != (format == "plain"):
            raise ValueError("k_scale and v_scale go with the quantised formats")
        if k_scale is not None:
            _need(k_scale, "k_scale", (num_pages, page_size), torch.float32, dev)
            _need(v_scale, "v_scale", (num_pages, page_size), torch.float32, dev)
        nseq, Hkv, max_pages = page_table.shape
        _need(page_table, "page_table", page_table.shape, torch.int32, dev)
        self.nseq, self.Hq, self.Hkv, self.dh = nseq, Hq, Hkv, dh
        self.page_size, self.num_pages, self.max_pages = page_size, num_pages, max_pages
        self.k_pages, self.v_pages, self.k_scale, self.v_scale = k_pages, v_pages, k_scale, v_scale
        self.page_table = page_table
        self.desc = B.make_cache(nseq=nseq, Hq=Hq, Hkv=Hkv, dh=dh, dtype=dtype, format=format, page_size=page_size,
                                 num_pages=num_pages, max_pages=max_pages, k_pages=k_pages, v_pages=v_pages,
                                 page_table=page_table, k_scale=k_scale, v_scale=v_scale, page_stride=strides[0],
                                 scale=scale, flags=flags)
        self._ws_bytes = B.criticalkv_decode_workspace_bytes(self.desc)   # also refuses a bad description
        self._ws = {}                    # workspaces by stream
        self._out_shape = (nseq, Hq, dh)
        # what attend's outputs look like: torch.empty_like costs half of torch.empty with a shape, a type and a device
        self._out_like = torch.empty(self._out_shape, dtype=self.torch_dtype, device=dev)
        self._lse_like = torch.empty((nseq, Hq), dtype=torch.float32, device=dev)
        self._ref = C.byref(self.desc)
        self._take_handle(handle, dev)
        self._decode, self._store = self._lib.criticalkv_decode, self._lib.criticalkv_cache_store
        self._load = self._lib.criticalkv_cache_load

    @classmethod
    def allocate(cls, *, nseq, Hq, Hkv, dh, dtype, rows, format="plain", page_size=64, device=0, **kw):
        """A cache with room for `rows` rows in every head, every page handed out."""
        dev = torch.device("cuda", device)
        cols = max(1, -(-rows // page_size))
        n = max(1, nseq * Hkv * cols)
        code = _CODE.get(format, _TORCH_DTYPE[dtype])
        pages = [torch.zeros((n, page_size, dh), dtype=torch.uint8 if code in _CODE.values() else code,
                             device=dev).view(code) for _ in range(2)]
        scales = [torch.zeros((n, page_size), dtype=torch.float32, device=dev) if format != "plain" else None
                  for _ in range(2)]
        table = torch.arange(nseq * Hkv * cols, dtype=torch.int32, device=dev).view(nseq, Hkv, cols)
        return cls(Hq=Hq, dtype=dtype, format=format, k_pages=pages[0], v_pages=pages[1], k_scale=scales[0],
                   v_scale=scales[1], page_table=table, **kw)

    def _kept(self):
        return self.k_pages, self.v_pages, self.k_scale, self.v_scale, self.page_table

    def new_lengths(self):
        """Lengths of an empty cache."""
        return torch.zeros((self.nseq, self.Hkv), dtype=torch.int32, device=self.device)

    def store(self, K, V, start, lens_out=None, *, idx=None, offsets=None, counts=None, stream=None):
        """Writes rows of K, V [nseq, Hkv, n, dh] behind row start[s, g] of every head and returns lens_out, which may
        be `start` (allocated when None).  All n rows, the first counts[s] of them, or with idx [nseq, idx_rows] and
        offsets [nseq, Hkv+1] the rows that CompressionSession.select chose.  K and V have the same strides: parts of one
        projection keep them when Rotary.rotate turns k in place (k_out=k)."""
        if lens_out is None:
            with self._allocating(stream):
                lens_out = torch.empty((self.nseq, self.Hkv), dtype=torch.int32, device=self.device)
        key = (K.dtype, K.shape, K.stride(), K.get_device(), V.dtype, V.shape, V.stride(), V.get_device(), start.dtype,
               start.shape, start.stride(), start.get_device(), lens_out.dtype, lens_out.shape, lens_out.stride(),
               lens_out.get_device(), _sig(idx), _sig(offsets), _sig(counts))
        n, idx_rows, strides = self._plans.get(key) or self._keep(
            key, self._describe_store(K, V, start, lens_out, idx, offsets, counts))
        if idx_rows == 0:      # no list, or an empty one, whose address could not be passed (n is 0 then)
            idx = offsets = None
        rc = self._store(
            self.handle, self._ref, K.data_ptr(), V.data_ptr(), n, strides, None if idx is None else idx.data_ptr(),
            None if offsets is None else offsets.data_ptr(), idx_rows, None if counts is None else counts.data_ptr(),
            start.data_ptr(), lens_out.data_ptr(), self._where(stream))
        if rc:
            self._fail(rc, "criticalkv_cache_store")
        return lens_out

    def _describe_store(self, K, V, start, lens_out, idx, offsets, counts):
        dev, shape = self.device, (self.nseq, self.Hkv)
        if K.dim() != 4:
            raise ValueError("K must be [nseq, Hkv, n, dh]")
        n = K.shape[2]
        _need(K, "K", (*shape, n, self.dh), self.torch_dtype, dev, dense=False)
        _need(V, "V", K.shape, self.torch_dtype, dev, dense=False)
        strides = _row_strides(K, "K")
        if strides != _row_strides(V, "V"):
            raise ValueError("K and V must have the same strides")
        _need(start, "start", shape, torch.int32, dev)
        _need(lens_out, "lens_out", shape, torch.int32, dev)
        idx_rows = 0
        if (idx is None) != (offsets is None):
            raise ValueError("idx and offsets go together")
        if idx is not None:
            if counts is not None:
                raise ValueError("counts cannot be combined with idx")
            idx_rows = idx.shape[-1]
            _need(idx, "idx", (self.nseq, idx_rows), torch.int32, dev)
            _need(offsets, "offsets", (self.nseq, self.Hkv + 1), torch.int32, dev)
        if counts is not None:
            _need(counts, "counts", (self.nseq,), torch.int32, dev)
        return (0 if idx is not None and idx_rows == 0 else n), idx_rows, B._strides(strides)

    def load(self, lens, n=None, K_out=None, V_out=None, *, align_right=False, stream=None):
        """Rows 0..min(lens, n)-1 of every head as K_out, V_out [nseq, Hkv, n, dh] (zeros where there is no row, when
        allocated here; left as they were in a caller's tensor).  align_right puts the last rows of a head at the end,
        as the compression step's valid_from = n - lens wants it."""
        if K_out is None or V_out is None:
            if n is None or K_out is not None or V_out is not None:
                raise ValueError("give n, or both K_out and V_out")
            with self._allocating(stream):
                K_out = torch.zeros((self.nseq, self.Hkv, n, self.dh), dtype=self.torch_dtype, device=self.device)
                V_out = torch.zeros_like(K_out)
        key = (n, lens.dtype, lens.shape, lens.stride(), lens.get_device(), K_out.dtype, K_out.shape, K_out.stride(),
               K_out.get_device(), V_out.dtype, V_out.shape, V_out.stride(), V_out.get_device())
        n, strides = self._plans.get(key) or self._keep(key, self._describe_load(lens, n, K_out, V_out))
        rc = self._load(self.handle, self._ref, lens.data_ptr(), n, strides, 1 if align_right else 0, K_out.data_ptr(),
                        V_out.data_ptr(), self._where(stream))
        if rc:
            self._fail(rc, "criticalkv_cache_load")
        return K_out, V_out

    def _describe_load(self, lens, n, K_out, V_out):
        dev = self.device
        _need(lens, "lens", (self.nseq, self.Hkv), torch.int32, dev)
        if K_out.dim() != 4 or (n is not None and n != K_out.shape[2]):
            raise ValueError("K_out must be [nseq, Hkv, n, dh]")
        n = K_out.shape[2]
        _need(K_out, "K_out", (self.nseq, self.Hkv, n, self.dh), self.torch_dtype, dev, dense=False)
        _need(V_out, "V_out", K_out.shape, self.torch_dtype, dev, dense=False)
        strides = _row_strides(K_out, "K_out")
        if strides != _row_strides(V_out, "V_out"):
            raise ValueError("K_out and V_out must have the same strides")
        return n, B._strides(strides)

    def workspace(self, stream=None):
        """The decode workspace of a stream (None: the current one): allocated there on first use and kept.  Calls on
        different streams have different ones, and while torch.cuda.graph captures a stream every call gets a new one from
        the graph's memory, so that neither two graphs nor a graph and other calls share any.  A capture that torch's
        allocator does not know of needs a `ws` argument that outlives the graph."""
        if stream is None:
            return self._workspace(_raw_stream(self._index))
        with self._allocating(stream):
            return self._workspace(self._on(stream))

    def _workspace(self, raw):
        """raw: the current stream."""
        if _current_device() == self._index:
            captured = _capturing()
        else:
            with torch.cuda.device(self._index):
                captured = _capturing()
        if captured:
            return torch.empty(self._ws_bytes, dtype=torch.uint8, device=self.device)
        ws = self._ws.get(raw)
        if ws is None:
            if len(self._ws) >= 64:      # streams that come and go
                self._ws.clear()
            ws = self._ws[raw] = torch.empty(self._ws_bytes, dtype=torch.uint8, device=self.device)
        return ws

    def attend(self, q, lens, out=None, lse=None, *, ws=None, stream=None):
        """Attention of one new token per sequence: q [nseq, Hq, dh] over the lens[s, g] rows of every head.  Returns
        (out [nseq, Hq, dh], lse float32 [nseq, Hq])."""
        key = (q.dtype, q.shape, q.stride(), q.get_device(), lens.dtype, lens.shape, lens.stride(), lens.get_device(),
               _sig(out), _sig(lse), _sig(ws))
        strides, size = self._plans.get(key) or self._keep(key, self._describe_attend(q, lens, out, lse, ws))
        raw = self._where(stream)
        if stream is None:
            out = torch.empty_like(self._out_like) if out is None else out
            lse = torch.empty_like(self._lse_like) if lse is None else lse
            ws = self._workspace(raw) if ws is None else ws
        else:
            with self._allocating(stream):
                out = torch.empty_like(self._out_like) if out is None else out
                lse = torch.empty_like(self._lse_like) if lse is None else lse
                ws = self._workspace(raw) if ws is None else ws
        rc = self._decode(self.handle, self._ref, q.data_ptr(), strides, lens.data_ptr(), out.data_ptr(), lse.data_ptr(),
                          ws.data_ptr(), size, raw)
        if rc:
            self._fail(rc, "criticalkv_decode")
        return out, lse

    def _describe_attend(self, q, lens, out, lse, ws):
        dev, shape = self.device, self._out_shape
        _need(q, "q", shape, self.torch_dtype, dev, dense=False)
        _need(lens, "lens", (self.nseq, self.Hkv), torch.int32, dev)
        if out is not None:
            _need(out, "out", shape, self.torch_dtype, dev)
        if lse is not None:
            _need(lse, "lse", shape[:2], torch.float32, dev)
        if ws is not None and (ws.device != dev or not ws.is_contiguous()):
            raise ValueError(f"ws must be contiguous on {dev}")
        return B._strides(_row_strides(q, "q")), self._ws_bytes if ws is None else ws.numel() * ws.element_size()
