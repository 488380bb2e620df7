"""Decode attention in 64 bits with bounds for each of the two kernels, narrow enough to see how many bits a weight has."""
from __future__ import annotations

import math

import torch

from cache_ref import DT, HALF_STEP, head_rows

STEP = 2.0 ** -23        # a float32 addition inside a matrix instruction (which may truncate); half of it on CUDA cores
WEIGHT_BITS = {          # relative rounding error of a weight in the product with the values
    ("tensor", "plain"): 2.0 ** -17,      # a bf16 (2^-9) and the bf16 of what is left (2^-9 of that), doubled
    ("tensor", "8-bit"): 2.0 ** -22,      # a half (2^-11) and the half of what is left (2^-11 of that)
    ("cuda", "plain"): 2.0 ** -24, ("cuda", "8-bit"): 2.0 ** -24}


def decode(q, values_k, values_v, table, lens, page_size, scale, fmt, dtype, kernel, vscale=None, moves=1):
    """out, lse in 64 bits and bounds on |kernel - out| and |kernel - lse|; kernel "tensor" (bf16) or "cuda".

    With weights w_i and relative errors d_i of theirs, out moves by sum w_i d_i (v_i - out) and lse by sum w_i d_i.
    d_i: the sum of a logit's dh products (dh additions, relative to sum |q||k|; queries of 8-bit pages as halves on the
    tensor cores: halves are multiples of 2^-24, so half a step is 2^-25; the largest element stands at 2^14 or above, which
    makes it 2^-39 of that each, but the scaling is by 2^100 at most, which makes it 2^-125 for tinier rows), four roundings relative to the logit (row scale, two factors, the
    difference to the maximum, which is at most twice the largest logit), 2^-22 of exp2 once and each time the running
    maximum moves (`moves`: of the order of ln n a warp, and three where warps, CTAs and parts meet).  Then the rounding of the weights in
    the second product, the additions over the rows (a quarter of them one behind the other at most, and 64 more where
    parts are joined) and the result's rounding.  Two halves: a product of weight and row scale loses 2^-40 of the largest
    such product at the least, times the code."""
    assert kernel in ("tensor", "cuda") and (kernel == "cuda" or dtype == "bf16")
    nseq, Hq, dh = q.shape
    Hkv = table.shape[1]
    G = Hq // Hkv
    out = torch.zeros((nseq, Hq, dh), dtype=torch.float64)
    lse = torch.full((nseq, Hq), -math.inf, dtype=torch.float64)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    coarse = WEIGHT_BITS[kernel, "plain" if fmt == "plain" else "8-bit"]
    for s in range(nseq):
        for g in range(Hkv):
            n = int(lens[s, g])
            if n == 0:
                continue
            K, V = (head_rows(v, table[s, g], n, page_size) for v in (values_k, values_v))
            qs, hs = q[s, g * G:(g + 1) * G].double().cpu(), slice(g * G, (g + 1) * G)
            logit = qs @ K.T * scale
            w = torch.softmax(logit, -1)
            out[s, hs] = w @ V
            lse[s, hs] = torch.logsumexp(logit, -1)
            d = (dh + 8) * STEP * abs(scale) * (qs.abs() @ K.abs().T) + 4 * STEP * logit.abs() + moves * 2.0 ** -22
            d = d + STEP * logit.abs().amax(-1, keepdim=True)
            if kernel == "tensor" and fmt != "plain":
                d = d + abs(scale) * (2.0 ** -39 * qs.abs().amax(-1, keepdim=True) + 2.0 ** -125) * K.abs().sum(-1)
            adds = (n / 4 + 64) * STEP
            for h in range(G):
                far = (V - out[s, g * G + h]).abs()
                tol[s, g * G + h] = (w[h] * d[h]) @ far * 1.02 + (coarse + adds) * (w[h] @ V.abs())
            tol[s, hs] += adds * out[s, hs].abs() + out[s, hs].abs() * HALF_STEP[dtype] + 1e-37
            if kernel == "tensor" and fmt != "plain":
                vs = head_rows(vscale.cpu().double()[..., None], table[s, g], n, page_size)[:, 0]
                tol[s, hs] += 2.0 ** -40 * (w * vs).amax(-1)[:, None] * (V.abs() / vs[:, None]).sum(0)
            tol_lse[s, hs] = (w * d).sum(-1) * 1.02 + adds + (lse[s, hs].abs() + 1.0) * STEP
    return out, lse, tol, tol_lse


def check(got, want, lens, G):
    """Every element within its bound (a NaN is not), zeros and -infinity where a head has no rows."""
    out, lse, tol, tol_lse = want
    o, l = got[0].cpu().double(), got[1].cpu().double()
    assert o.shape == out.shape and l.shape == lse.shape
    assert bool(((o - out).abs() <= tol).all())
    empty = (lens == 0).repeat_interleave(G, dim=1)
    assert bool((o[empty] == 0).all()) and bool((l[empty] == -math.inf).all())
    assert bool(((l - lse).abs() <= tol_lse)[~empty].all())
