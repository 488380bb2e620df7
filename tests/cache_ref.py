"""Plain forms of rotary positions, the paged cache and decode attention for the tests, in 64 bits unless stated."""
from __future__ import annotations

import math

import numpy as np
import torch

TOP = {"e4m3": 448.0, "int8": 127.0}
CODE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}       # largest relative rounding error of a stored result


def rope(x, pos, freq, layout, factor=1.0):
    """x [nseq, H, T, dh], pos [nseq, T] int, freq [rot/2]: CPU tensors -> float64."""
    y = x.double().clone()
    h = freq.numel()
    angle = pos.double()[:, None, :, None] * freq
    c, s = factor * torch.cos(angle), factor * torch.sin(angle)
    ia = torch.arange(h) if layout == "half" else 2 * torch.arange(h)
    ib = ia + (h if layout == "half" else 1)
    a, b = x.double()[..., ia], x.double()[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    return y


def quantise(rows, fmt):
    """Codes and scales of CPU rows [..., dh] by the documented rule, every operation a float32 one (numpy's are IEEE)."""
    x = rows.float().numpy()
    with np.errstate(invalid="ignore", over="ignore"):
        top = np.abs(x).max(-1)                               # NaN where the row has one
        scale = (top / np.float32(TOP[fmt])).astype(np.float32)
        scale = np.where(scale < np.float32(2.0 ** -100), np.float32(2.0 ** -100), scale)
        over = np.isfinite(top) & np.isinf(scale * np.float32(TOP[fmt]))
        scale = np.where(over, np.nextafter(scale, np.float32(0.0)), scale)
        y = x * (np.float32(1.0) / scale)[..., None]
    y = torch.from_numpy(np.ascontiguousarray(y))
    if fmt == "e4m3":
        code = y.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    else:
        code = torch.nan_to_num(y).round().clamp(-127, 127).to(torch.int8)
    return code, torch.from_numpy(scale)


def stored(pages, scale, fmt):
    """The values the pages stand for, float64 CPU [num_pages, page_size, dh]."""
    x = pages.cpu().float().double()
    return x if fmt == "plain" else x * scale.cpu().double()[..., None]


def head_rows(values, table_row, n, page_size):
    """Rows 0..n-1 of one head."""
    i = torch.arange(n)
    return values[table_row.long().cpu()[i // page_size], i % page_size]


def decode(q, values_k, values_v, table, lens, page_size, scale, fmt, dtype, vscale=None):
    """out, lse in 64 bits and a bound on |kernel - out| and |kernel - lse| for each element.

    The bound counts, for weights w_i (sum 1) over rows v_i: dh + 8 float32 roundings of a logit's products (eps_s, on
    sum |q||k| * scale), 4 float32 roundings of exp2 and of the scaling by log2(e) (relative to the largest logit),
    which both move a weight by a relative error and the result by at most twice that times sum w|v|; the rounding of
    a weight for the tensor core (16 bits for plain pages, 2^-11 for 8-bit pages and 2^-24 of the largest weight times
    scale where that is coarser); float32 additions of the values; the rounding of the result."""
    nseq, Hq, dh = q.shape
    Hkv = table.shape[1]
    G = Hq // Hkv
    out = torch.zeros((nseq, Hq, dh), dtype=torch.float64)
    lse = torch.full((nseq, Hq), -math.inf, dtype=torch.float64)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    eps = 2.0 ** -23
    for s in range(nseq):
        for g in range(Hkv):
            n = int(lens[s, g])
            if n == 0:
                continue
            K, V = (head_rows(v, table[s, g], n, page_size) for v in (values_k, values_v))
            qs = q[s, g * G:(g + 1) * G].double().cpu()
            logit = qs @ K.T * scale
            w = torch.softmax(logit, -1)
            hs = slice(g * G, (g + 1) * G)
            out[s, hs] = w @ V
            lse[s, hs] = torch.logsumexp(logit, -1)
            mass = w @ V.abs()
            ds = eps * ((dh + 8) * (qs.abs() @ K.abs().T * abs(scale)).amax(-1) + 4 * logit.abs().amax(-1) + 4)
            coarse = 2.0 ** -16 if fmt == "plain" else 2.0 ** -11
            tol[s, hs] = mass * (2 * ds + coarse + (n + 64) * eps)[:, None] + out[s, hs].abs() * HALF_STEP[dtype] + 1e-37
            if fmt != "plain" and dtype == "bf16":
                vs = head_rows(vscale.cpu().double()[..., None], table[s, g], n, page_size)[:, 0]
                tol[s, hs] += (n * 2.0 ** -24 * (w * vs).amax(-1))[:, None] * (V.abs() / vs[:, None]).amax(0)
            tol_lse[s, hs] = ds + (n + 64) * eps + lse[s, hs].abs() * 2.0 ** -23
    return out, lse, tol, tol_lse
