"""Pages in 4 bits a value for the tests: the documented rule in numpy's float32, what the codes stand for in 64 bits, and a
cache whose unused rows are garbage."""
from __future__ import annotations

import math

import numpy as np
import torch

import cache_ref as R
import decode_bounds
from canary_util import Guarded
from paper_2502_03805_b200 import PagedCache

LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def encode(y):
    """Codes 0..15 of float32 numbers: the nearest of LEVELS, the one with an even code where two are as near."""
    size = np.abs(y).astype(np.float64)
    code = np.zeros(y.shape, np.uint8)
    middles = (LEVELS[:-1] + LEVELS[1:]).numpy() / 2
    for i, m in enumerate(middles):
        code += ((size > m) | ((size == m) & (i % 2 == 1))).astype(np.uint8)      # from level i to i + 1
    return code | (np.signbit(y).astype(np.uint8) << 3)


def quantise(rows):
    """Packed codes, group scales (e4m3) and row scales of CPU rows [..., dh]."""
    f = np.float32
    x = rows.float().numpy()
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        top = np.abs(x).max(-1)
        scale = (top / f(2688)).astype(f)
        scale = np.where(scale < f(2.0 ** -100), f(2.0 ** -100), scale)
        over = np.isfinite(top) & np.isinf(scale * f(2688))
        scale = np.where(over, np.nextafter(scale, f(0.0)), scale)
        r = (f(1.0) / scale)[..., None]
        groups = x.reshape(*x.shape[:-1], x.shape[-1] // 16, 16)
        s = (np.abs(groups).max(-1) * r) * (f(1.0) / f(6.0))
        s = np.where(np.isfinite(top)[..., None], s, f(0.0)).astype(f)
        g = torch.from_numpy(np.minimum(s, f(448.0))).to(torch.float8_e4m3fn)
        gf = g.float().numpy()
        factor = np.where(gf > 0, r / np.where(gf > 0, gf, f(1.0)), f(0.0)).astype(f)[..., None]
        y = np.where(factor == 0, f(0.0), groups * factor).reshape(x.shape)
    code = encode(y)
    return torch.from_numpy(code[..., 0::2] | (code[..., 1::2] << 4)), g, torch.from_numpy(scale)


def values(pages, groups, scale):
    """What stored rows stand for, float64 on the CPU."""
    two = pages.cpu().long()
    code = torch.stack([two & 15, two >> 4], -1).flatten(-2)
    x = LEVELS[code & 7] * torch.where(code > 7, -1.0, 1.0)
    x = x * groups.cpu().float().double().repeat_interleave(16, -1)
    return x * scale.cpu().double()[..., None]


class FourBit:
    """Pages in guarded buffers, garbage (NaN scales) wherever no row is stored; the attributes of the tests' other cache."""
    fmt = "e2m1"

    def __init__(self, *, nseq, Hq, Hkv, dh, dtype, page, cols, seed=0, spare=2, interleave=False, flags=0, scale=0.0):
        self.dtype, self.page, self.dh, self.Hkv, self.Hq = dtype, page, dh, Hkv, Hq
        n = nseq * Hkv * cols + spare
        self.table = torch.randperm(n, generator=torch.Generator().manual_seed(seed))[:nseq * Hkv * cols].view(
            nseq, Hkv, cols).to(torch.int32)
        if interleave:
            pool = Guarded((n, 2, page, dh // 2), torch.uint8, fill=0x7f)
            self.k, self.v, self.guards = pool.t[:, 0], pool.t[:, 1], [pool]
        else:
            self.guards = [Guarded((n, page, dh // 2), torch.uint8, fill=0x7f) for _ in range(2)]
            self.k, self.v = (x.t for x in self.guards)
        s = [Guarded((n, page), torch.float32, fill=math.nan) for _ in range(2)]
        g = [Guarded((n, page, dh // 16), torch.uint8, fill=0x7f) for _ in range(2)]
        self.guards += s + g
        self.ks, self.vs = s[0].t, s[1].t
        self.kg, self.vg = (x.t.view(torch.float8_e4m3fn) for x in g)
        self.table_dev = self.table.cuda()
        self.c = self.other(flags=flags, scale=scale)

    def other(self, table=None, **kw):
        return PagedCache(Hq=self.Hq, dtype=self.dtype, format="e2m1", k_pages=self.k, v_pages=self.v, k_scale=self.ks,
                          v_scale=self.vs, k_group_scale=self.kg, v_group_scale=self.vg,
                          page_table=self.table_dev if table is None else table, **kw)

    def parts(self):
        """Codes, group scales and row scales of K and of V."""
        return (self.k, self.kg, self.ks), (self.v, self.vg, self.vs)

    def fill(self, lens, seed, spread=1.0):
        """Random rows in every head, quantised on the CPU."""
        g = torch.Generator().manual_seed(seed)
        for s in range(lens.shape[0]):
            for h in range(self.Hkv):
                n = int(lens[s, h])
                if n:
                    rows = [(torch.randn(n, self.dh, generator=g) * torch.exp(spread * torch.randn(n, 1, generator=g))).to(
                        R.DT[self.dtype]) for _ in range(2)]
                    self.put(s, h, torch.arange(n), rows)
        return self

    def put(self, s, h, at, rows):
        """Rows (K and V) written to places `at` of a head, not by the library."""
        page, slot = self.table[s, h].long()[at // self.page].cuda(), (at % self.page).cuda()
        for x, (code, group, scale) in zip(rows, self.parts()):
            c, g, sc = quantise(x)
            code[page, slot] = c.cuda()
            group.view(torch.uint8)[page, slot] = g.view(torch.uint8).cuda()
            scale[page, slot] = sc.cuda()

    def values(self):
        return tuple(values(*p) for p in self.parts())

    def bits(self):
        return [x.contiguous().view(torch.uint8).cpu() for p in self.parts() for x in p]

    def intact(self):
        return all(g.intact() for g in self.guards)


def expect_store(cache, before, K, V, rows_of, start):
    """The arrays of `before` (bits) with the rows rows_of(s, h) of K, V written behind start."""
    want = [b.clone() for b in before]
    cap = cache.table.shape[2] * cache.page
    shapes = [p[i].shape for p in cache.parts() for i in range(3)]
    for s in range(K.shape[0]):
        for h in range(cache.Hkv):
            src = torch.as_tensor(rows_of(s, h), dtype=torch.long)
            to = int(start[s, h]) + torch.arange(len(src))
            keep = (to >= 0) & (to < cap) & (src >= 0) & (src < K.shape[2])
            src, to = src[keep], to[keep]
            page, slot = cache.table[s, h].long()[to // cache.page], to % cache.page
            for j, x in enumerate((K[s, h, src], V[s, h, src])):
                code, group, scale = quantise(x)
                want[3 * j].view(shapes[3 * j])[page, slot] = code
                want[3 * j + 1].view(shapes[3 * j + 1])[page, slot] = group.view(torch.uint8)
                want[3 * j + 2].view(torch.float32).view(shapes[3 * j + 2])[page, slot] = scale
    return want


def attention(q, cache, lens, scale, kernel, table=None, moves=16):
    """out, lse in 64 bits and bounds on |kernel - out| and |kernel - lse|, as decode_bounds.decode has them; kernel "tensor" or
    "cuda" (whose bounds are those of 8-bit pages).

    Tensor cores: the products of codes and group scales are exact; a query element is one half (bf16: exact but for 2^-39 of the
    row's largest) or the sum of two (float32: half a step of the second, 2^-24 of the element, besides); a weight is the sum of
    two halves (2^-22) and loses 2^-36 of the largest product of a weight and a row scale at the least, times code and group
    scale.  `moves`: how often the references move, each time 2^-22 of exp2."""
    D, G = decode_bounds, q.shape[1] // cache.Hkv
    K, V = cache.values()
    table = cache.table if table is None else table
    if kernel == "cuda":
        return D.decode(q, K, V, table, lens, cache.page, scale, "e2m1", cache.dtype, kernel, cache.vs, moves)
    out = torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    vs_all = cache.vs.cpu().double()[..., None]
    for s in range(q.shape[0]):
        for g in range(cache.Hkv):
            n = int(lens[s, g])
            if n == 0:
                continue
            k, v, vs = (R.head_rows(x, table[s, g], n, cache.page) for x in (K, V, vs_all))
            qs, hs = q[s, g * G:(g + 1) * G].double().cpu(), slice(g * G, (g + 1) * G)
            logit = qs @ k.T * scale
            w = torch.softmax(logit, -1)
            out[s, hs], lse[s, hs] = w @ v, torch.logsumexp(logit, -1)
            size = abs(scale) * (qs.abs() @ k.abs().T)
            d = (cache.dh + 8 + (1 if cache.dtype == "f32" else 0)) * D.STEP * size + 4 * D.STEP * logit.abs() + moves * 2.0 ** -22
            d = d + D.STEP * logit.abs().amax(-1, keepdim=True)
            d = d + abs(scale) * (2.0 ** -39 * qs.abs().amax(-1, keepdim=True) + 2.0 ** -125) * k.abs().sum(-1)
            adds = (n / 4 + 64) * D.STEP
            for h in range(G):
                far = (v - out[s, g * G + h]).abs()
                tol[s, g * G + h] = (w[h] * d[h]) @ far * 1.02 + (2.0 ** -22 + adds) * (w[h] @ v.abs())
            tol[s, hs] += adds * out[s, hs].abs() + out[s, hs].abs() * R.HALF_STEP[cache.dtype] + 1e-37
            tol[s, hs] += 2.0 ** -36 * (w * vs[:, 0]).amax(-1)[:, None] * (v.abs() / vs).sum(0)
            tol_lse[s, hs] = (w * d).sum(-1) * 1.02 + adds + (lse[s, hs].abs() + 1.0) * D.STEP
    return out, lse, tol, tol_lse
