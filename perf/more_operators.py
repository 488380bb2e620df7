"""Decoding on caches that are smaller or read in part: what is measured, and the plain form of each operator.

Five passes next to the ones of a serving loop that the compression step is followed by:

  append     new tokens' queries and keys rotated, their keys and values written into the paged cache
  store4     the rows a selection kept written into pages of 4 bits a value, and read back
  attend4    attention of one new token over pages of 4 bits a value
  summarise  the largest and smallest key of every page, in 8 bits
  sparse     attention of one new token over the pages that score best against it

A case is a dict of plain values; prepare() makes its inputs on the GPU from a seed, run() makes one pass.  With `own`
false run() computes the operators with elementary torch operations in 32 bits (angles in 64); with `own` true it calls
the library.

4 bits a value ("e2m1"): 1 sign, 2 exponent, 1 fraction bit (0, 0.5, 1, 1.5, 2, 3, 4, 6), two to a byte, the earlier
element in the low half.  A row has a float32 scale S, each of its groups of 16 elements an e4m3 scale s; a code stands for
(code * s) * S.
"""
import math
import random

import numpy as np
import torch

own = False
_handle = None       # the library handle a program keeps for its lifetime

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_TOP = {"e4m3": 448.0, "int8": 127.0}
_CODE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8, "e2m1": torch.uint8}
_LEAST = 2.0 ** -100     # smallest scale of a stored row, of a page's summary and of a query's codes
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---- cases -------------------------------------------------------------------------------------------------------
def listed():
    head = dict(Hq=32, Hkv=8, dh=128, dtype="bf16")          # 32 query heads on 8 KV heads, as the 32-layer workload
    return [
        # one new token of one sequence, far into a long context
        dict(name="append one token", op="append", nseq=1, T=1, rot=128, layout="half", page=64, format="plain", at=13107,
             pos=131000, **head),
        # one new token of each of 61 sequences, half of a 64-wide head rotated in interleaved pairs, 4 bits a value
        dict(name="append 61 tokens 4 bits", op="append", nseq=61, T=1, Hq=8, Hkv=2, dh=64, dtype="bf16", rot=32,
             layout="interleaved", page=16, format="e2m1", at=777, pos=5000),
        # a whole prompt of the headline length
        dict(name="append prompt 32768", op="append", nseq=1, T=32768, rot=128, layout="half", page=64, format="plain", at=0,
             pos=0, **head),
        # the rows an adaptive selection kept (20 % of 32768 per head on average), 8 layers at once
        dict(name="store kept rows 4 bits", op="store4", nseq=8, n=32768, kept=6553, page=64, at=0, **head),
        # the new tokens of 16 sequences
        dict(name="store 16 tokens 4 bits", op="store4", nseq=16, n=1, kept=0, page=64, at=6553, **head),
        # one sequence, a short cache: latency
        dict(name="attend one, 819 rows", op="attend4", nseq=1, rows=819, spread=0.5, page=64, **head),
        # 32 sequences on caches an adaptive budget compressed to 20 % of 32768
        dict(name="attend 32, kept rows", op="attend4", nseq=32, rows=6553, spread=0.8, page=64, **head),
        # float32 model with a 64-wide head, a few sequences, odd lengths, one head empty
        dict(name="attend 5, float32", op="attend4", nseq=5, rows=1237, spread=1.0, page=16, Hq=8, Hkv=2, dh=64, dtype="f32"),
        # a long prompt's pages
        dict(name="summarise 131072 rows", op="summarise", nseq=1, rows=131072, spread=0.0, page=64, format="plain", new=0,
             **head),
        # the last page of every head after a decode step
        dict(name="summarise last pages", op="summarise", nseq=16, rows=6553, spread=0.8, page=64, format="e4m3", new=1, **head),
        # one sequence, 64 of 2048 pages
        dict(name="sparse one, 131072 rows", op="sparse", nseq=1, rows=131072, spread=0.0, page=64, format="plain", pages=64,
             **head),
        # 32 sequences of about 32768 rows on 4 bits a value, 32 pages each
        dict(name="sparse 32, 4 bits", op="sparse", nseq=32, rows=32768, spread=0.3, page=64, format="e2m1", pages=32, **head),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges the listed ones stand for, no larger than the largest listed one of its operator."""
    c = _draw(rng)
    while work(c)["bytes"] > max(work(x)["bytes"] for x in listed() if x["op"] == c["op"]):
        c = _draw(rng)
    return c


def _draw(rng):
    op = rng.choice(["append", "append", "store4", "attend4", "attend4", "summarise", "sparse", "sparse"])
    Hkv = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 4, 5, 8])
    dh = rng.choice([64, 128])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    c = dict(op=op, Hq=Hkv * G, Hkv=Hkv, dh=dh, dtype=dtype, page=rng.choice([16, 32, 64, 128]))
    if op == "append":
        T = _log(rng, 1, 32768)
        nseq = _log(rng, 1, max(1, min(64, 32768 // T)))
        # a float32 key that differs in its last bit may take the next code: such rows say nothing about a kernel
        form = "plain" if dtype == "f32" else rng.choice(["plain", "e4m3", "int8", "e2m1"])
        return dict(c, nseq=nseq, T=T, rot=rng.choice([dh, dh // 2, dh // 4]), layout=rng.choice(["half", "interleaved"]),
                    format=form, at=rng.randrange(200), pos=rng.randrange(131072 - T + 1))
    if op == "store4":
        n = _log(rng, 1, 32768)
        nseq = _log(rng, 1, max(1, min(64, 131072 // n)))
        kept = rng.choice([0, max(1, n // 5)]) if n >= 8 else 0
        return dict(c, nseq=nseq, n=n, kept=kept, at=0 if kept else rng.randrange(200))
    if op == "attend4":
        rows = _log(rng, 16, 65536)
        nseq = _log(rng, 1, max(1, min(64, 131072 // rows)))
        return dict(c, nseq=nseq, rows=rows, spread=rng.choice([0.0, 0.5, 0.8, 1.0]))
    c["format"] = rng.choice(["plain", "e4m3", "int8", "e2m1"])
    rows = _log(rng, 64, 131072)
    nseq = _log(rng, 1, max(1, min(32, 131072 // rows)))
    c.update(nseq=nseq, rows=rows, spread=rng.choice([0.0, 0.3, 0.8]))
    if op == "summarise":
        return dict(c, new=rng.choice([0, 0, 1, 100]))
    return dict(c, pages=_log(rng, 2, 128))


def _ragged(nseq, Hkv, mean, spread, most):
    """Row counts [nseq][Hkv] of the heads, the same for every seed; with spread 1 the last head is empty."""
    r = random.Random("%d %d %d %r" % (nseq, Hkv, mean, spread))
    at = [[max(0, min(most, round(mean * (1 + spread * r.uniform(-1, 1))))) for _ in range(Hkv)] for _ in range(nseq)]
    if spread >= 1.0:
        at[-1][-1] = 0
    return at


def _counts(c):
    """Rows of every head of a case: written by `append` and `store4`, held for the others."""
    if c["op"] == "append":
        return [[c["T"]] * c["Hkv"] for _ in range(c["nseq"])]
    if c["op"] == "store4":
        if not c["kept"]:
            return [[c["n"]] * c["Hkv"] for _ in range(c["nseq"])]
        return _ragged(c["nseq"], c["Hkv"], c["kept"], 0.8, c["n"])
    return _ragged(c["nseq"], c["Hkv"], c["rows"], c["spread"], 2 * c["rows"])


def _format(c):
    return c.get("format", "e2m1")


# ---- inputs ------------------------------------------------------------------------------------------------------
def _frequencies(c):
    i = np.arange(c["rot"] // 2, dtype=np.float64)
    return 500000.0 ** (-2.0 * i / c["rot"])


def _rows_like_cache(g, shape, dtype, keys):
    """Rows as a cache holds them: keys with a few large channels, neighbours alike; values whose norm varies from token to
    token."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    if keys:
        if len(shape) == 3:                       # a pool: the rows of a page share a direction
            x += torch.randn((shape[0], 1, shape[2]), generator=g, device="cuda")
        x[..., 3::32] *= 8.0
    else:
        x *= torch.exp(torch.randn(shape[:-1] + (1,), generator=g, device="cuda"))
    return x.to(dtype)


def _table(c, counts, g, spare=3):
    """Page table [nseq, Hkv, columns] over a shuffled pool, -1 behind a head's last page, and the pool's size."""
    need = torch.tensor(counts, device="cuda").add(c["page"] - 1).div(c["page"], rounding_mode="floor")
    most, total = max(1, int(need.max())), int(need.sum())
    pages = torch.randperm(total + spare, generator=g, device="cuda")[:total].to(torch.int32)
    used = torch.arange(most, device="cuda") < need[..., None]
    table = torch.full(used.shape, -1, dtype=torch.int32, device="cuda")
    table[used] = pages
    return table, total + spare


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt, form = _DT[c["dtype"]], _format(c)
    s = dict(case=c)
    counts, at = _counts(c), c.get("at", 0)
    s["table"], pages = _table(c, [[x + at for x in row] for row in counts], g)
    pool = (pages, c["page"], c["dh"])
    held = pool[:2] + (c["dh"] // 2,) if form == "e2m1" else pool
    counts_t = torch.tensor(counts, dtype=torch.int32, device="cuda")
    for name in ("k", "v"):
        s[name + "_pages"], s[name + "_scale"], s[name + "_group"] = None, None, None
    if c["op"] in ("append", "store4"):
        for name in ("k", "v"):
            s[name + "_pages"] = torch.zeros(held, device="cuda").to(_CODE.get(form, dt))
            s[name + "_scale"] = torch.zeros(pool[:2], device="cuda") if form != "plain" else None
            s[name + "_group"] = torch.zeros(pool[:2] + (c["dh"] // 16,), device="cuda").to(torch.float8_e4m3fn) if form == "e2m1" else None
        s["start"] = torch.full((c["nseq"], c["Hkv"]), at, dtype=torch.int32, device="cuda")
        s["lens"] = torch.zeros_like(s["start"])
    if c["op"] == "append":
        both = torch.randn((c["nseq"], c["T"], c["Hq"] + 2 * c["Hkv"], c["dh"]), generator=g, device="cuda").to(dt)
        parts = both.split([c["Hq"], c["Hkv"], c["Hkv"]], dim=2)                 # parts of one projection's output
        s["q"], s["k"], s["v"] = (x.transpose(1, 2) for x in parts)
        first = torch.randint(0, 64, (c["nseq"], 1), generator=g, device="cuda", dtype=torch.int32)
        s["pos"] = (c["pos"] + first + torch.arange(c["T"], device="cuda", dtype=torch.int32)).contiguous()
        s["freq"] = torch.from_numpy(_frequencies(c)).cuda()
        s["q_out"] = torch.empty((c["nseq"], c["Hq"], c["T"], c["dh"]), dtype=dt, device="cuda")
        s["columns"] = c["T"]
        return s
    if c["op"] == "store4":
        src = (c["nseq"], c["Hkv"], c["n"], c["dh"])
        s["K"], s["V"] = _rows_like_cache(g, src, dt, True), _rows_like_cache(g, src, dt, False)
        s["idx"] = s["offsets"] = None
        s["columns"] = max(max(row) for row in counts)
        if c["kept"]:
            order = torch.rand(src[:3], generator=g, device="cuda").argsort(-1).argsort(-1)
            flat = (order < counts_t[..., None]).nonzero()[:, 2].to(torch.int32)
            total = counts_t.sum(1)
            most = int(total.max())
            s["idx"] = torch.full((c["nseq"], most), -1, dtype=torch.int32, device="cuda")
            s["idx"][torch.arange(most, device="cuda") < total[:, None]] = flat
            s["offsets"] = torch.nn.functional.pad(counts_t.cumsum(1), (1, 0)).to(torch.int32)
            s["total"] = [sum(row) for row in counts]
        return s
    s["lens"] = counts_t
    for name in ("k", "v"):
        x = _rows_like_cache(g, pool, dt, name == "k")
        if form == "plain":
            s[name + "_pages"] = x
        elif form == "e2m1":
            s[name + "_pages"], s[name + "_group"], s[name + "_scale"] = _quantise4(x)
        else:
            code, s[name + "_scale"] = _quantise8(x, form)
            s[name + "_pages"] = code
    s["columns"] = max(1, max(max(row) for row in counts))
    if c["op"] == "summarise":
        s["codes"] = torch.zeros((pages, 2, c["dh"]), dtype=torch.int8, device="cuda")
        s["page_scale"] = torch.zeros((pages,), device="cuda")
        s["from"] = (counts_t - c["new"]).clamp(min=0) if c["new"] else None
        return s
    # queries whose logits have a standard deviation near 2.5 over these keys
    s["q"] = (torch.randn((c["nseq"], c["Hq"], c["dh"]), generator=g, device="cuda") * (2.5 / math.sqrt(6.0))).to(dt)
    if c["op"] == "sparse":
        s["from"] = None
        s["codes"] = torch.zeros((pages, 2, c["dh"]), dtype=torch.int8, device="cuda")
        s["page_scale"] = torch.zeros((pages,), device="cuda")
        _summarise_plain(s)
    return s


# ---- plain forms -------------------------------------------------------------------------------------------------
def _quantise8(x, form):
    """Codes and scales of rows: scale = largest magnitude / largest code, code = value * (1 / scale) rounded."""
    y = x.float()
    top = y.abs().amax(-1)
    scale = (top / torch.full_like(top, _TOP[form])).clamp(min=_LEAST)
    y = y * scale.reciprocal()[..., None]
    if form == "e4m3":
        return y.clamp(-448.0, 448.0).to(torch.float8_e4m3fn), scale
    return y.round().clamp(-127.0, 127.0).to(torch.int8), scale


def _quantise4(x):
    """Packed codes, e4m3 scales of the groups and float32 scales of the rows."""
    y = x.float()
    top = y.abs().amax(-1)
    scale = (top / torch.full_like(top, 2688.0)).clamp(min=_LEAST)               # 448 * 6
    inverse = scale.reciprocal()[..., None]
    groups = y.unflatten(-1, (-1, 16))
    group = (groups.abs().amax(-1) * inverse * torch.tensor(1.0 / 6.0, device=y.device)).clamp(max=448.0).to(torch.float8_e4m3fn)
    s = group.float()
    y = (groups * torch.where(s > 0, inverse.expand_as(s) / s, torch.zeros_like(s))[..., None]).flatten(-2)
    size = y.abs().clamp(max=6.0)
    step = torch.where(size < 2.0, 0.5, torch.where(size < 4.0, 1.0, 2.0))
    size = torch.round(size / step) * step
    code = torch.where(size < 2.0, size * 2.0, torch.where(size < 4.0, size + 2.0, size * 0.5 + 4.0)).to(torch.uint8)
    code = code | (torch.signbit(y).to(torch.uint8) << 3)
    return code[..., 0::2] | (code[..., 1::2] << 4), group, scale


def _rows_plain(s, name, slot):
    """Stored rows `slot` (page * page_size + row) as float32."""
    c, form = s["case"], _format(s["case"])
    pages = s[name + "_pages"]
    if form == "plain":
        return pages.view(-1, c["dh"])[slot].float()
    scale = s[name + "_scale"].view(-1)[slot][..., None]
    if form == "e4m3":
        return pages.view(torch.uint8).view(-1, c["dh"])[slot].view(torch.float8_e4m3fn).float() * scale
    if form == "int8":
        return pages.view(-1, c["dh"])[slot].float() * scale
    level = torch.tensor(_LEVELS + tuple(-x for x in _LEVELS), device="cuda")
    two = pages.view(-1, c["dh"] // 2)[slot].int()
    code = torch.stack([level[two & 15], level[two >> 4]], -1).flatten(-2)
    group = s[name + "_group"].view(torch.uint8).view(-1, c["dh"] // 16)[slot].view(torch.float8_e4m3fn).float()
    return (code.unflatten(-1, (-1, 16)) * group[..., None]).flatten(-2) * scale


def _write_plain(s, name, slot, x):
    c, form = s["case"], _format(s["case"])
    pages = s[name + "_pages"]
    if form == "plain":
        pages.view(-1, c["dh"])[slot] = x
        return
    if form == "e2m1":
        code, group, scale = _quantise4(x)
        s[name + "_group"].view(torch.uint8).view(-1, c["dh"] // 16)[slot] = group.view(torch.uint8)
    else:
        code, scale = _quantise8(x, form)
        code, pages = code.view(torch.uint8), pages.view(torch.uint8)
    pages.view(-1, code.shape[-1])[slot] = code
    s[name + "_scale"].view(-1)[slot] = scale


def _slots(s, seq, head, row):
    page = s["case"]["page"]
    return s["table"][seq, head, row // page].clamp(min=0).long() * page + row % page


def _every_row(s, n):
    """Sequence, head and number of rows 0..n-1 of every head."""
    c = s["case"]
    row = torch.arange(n, device="cuda").expand(c["nseq"], c["Hkv"], n)
    seq = torch.arange(c["nseq"], device="cuda")[:, None, None].expand_as(row)
    return seq, torch.arange(c["Hkv"], device="cuda")[None, :, None].expand_as(row), row


def _turn_plain(s, x):
    c, h = s["case"], s["case"]["rot"] // 2
    angle = s["pos"].double()[:, None, :, None] * s["freq"]
    cos, sin = angle.cos().float(), angle.sin().float()
    y = x.float()
    if c["layout"] == "half":
        a, b = y[..., :h], y[..., h:2 * h]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin, y[..., 2 * h:]], -1)
    else:
        a, b = y[..., 0:2 * h:2], y[..., 1:2 * h:2]
        z = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        y = torch.cat([z, y[..., 2 * h:]], -1)
    return y.to(x.dtype)


def _read_back(s):
    """The rows that were written as dense tensors, zeros where a head has fewer than others."""
    seq, head, row = _every_row(s, s["columns"])
    row = row + s["start"][..., None]
    there = (row < s["lens"][..., None])[..., None]
    slot = _slots(s, seq, head, row)
    dt = _DT[s["case"]["dtype"]]
    return tuple(torch.where(there, _rows_plain(s, name, slot).to(dt), torch.zeros((), dtype=dt, device="cuda")) for name in ("k", "v"))


def _append_plain(s):
    c = s["case"]
    q_out = _turn_plain(s, s["q"])
    seq, head, row = _every_row(s, c["T"])
    slot = _slots(s, seq, head, row + s["start"][..., None])
    _write_plain(s, "k", slot, _turn_plain(s, s["k"]))
    _write_plain(s, "v", slot, s["v"])
    lens = s["start"] + c["T"]
    if c["format"] == "plain":
        return q_out, s["k_pages"], s["v_pages"], lens
    dt = _DT[c["dtype"]]
    return q_out, _rows_plain(s, "k", slot).to(dt), _rows_plain(s, "v", slot).to(dt), lens


def _store4_plain(s):
    c = s["case"]
    if s["idx"] is None:
        seq, head, row = _every_row(s, c["n"])
        src = row
    else:
        counts = s["offsets"].diff(dim=1)
        flat = torch.repeat_interleave(torch.arange(counts.numel(), device="cuda"), counts.flatten(),
                                       output_size=sum(s["total"]))
        seq, head = flat // c["Hkv"], flat % c["Hkv"]
        before = torch.nn.functional.pad(counts.flatten().cumsum(0), (1, 0))
        row = torch.arange(sum(s["total"]), device="cuda") - before[flat]
        src = s["idx"][seq, s["offsets"][seq, head] + row].long()
    slot = _slots(s, seq, head, row + s["start"][seq, head])
    for name in ("k", "v"):
        _write_plain(s, name, slot, s[name.upper()][seq, head, src])
    s["lens"].copy_(s["start"] + (c["n"] if s["idx"] is None else s["offsets"].diff(dim=1)))
    return (*_read_back(s), s["lens"])


def _attention_plain(s, K, V, there):
    """q [nseq, Hq, dh] over float32 rows K, V [nseq, Hkv, n, dh], of which there [nseq, Hkv, n] exist."""
    c = s["case"]
    q = s["q"].float().view(c["nseq"], c["Hkv"], -1, c["dh"])
    logit = (q @ K.transpose(-1, -2) * (1.0 / math.sqrt(c["dh"]))).masked_fill(~there[:, :, None], -math.inf)
    none = ~there.any(-1)[..., None, None]
    top = logit.amax(-1, keepdim=True)
    w = torch.exp(logit - top.masked_fill(none, 0.0))
    total = w.sum(-1, keepdim=True)
    out = (w @ V.masked_fill(~there[..., None], 0.0) / total).masked_fill(none, 0.0)
    lse = (top + torch.log(total)).masked_fill(none, -math.inf)
    return out.to(s["q"].dtype).view(c["nseq"], c["Hq"], c["dh"]), lse.view(c["nseq"], c["Hq"])


def _attend4_plain(s):
    seq, head, row = _every_row(s, s["columns"])
    slot = _slots(s, seq, head, row)
    return _attention_plain(s, _rows_plain(s, "k", slot), _rows_plain(s, "v", slot), row < s["lens"][..., None])


def _summarise_plain(s):
    """Codes [pages, 2, dh] (largest, smallest) and scale of every page that holds a row from s["from"] on."""
    c = s["case"]
    table, lens = s["table"], s["lens"][..., None]
    column = torch.arange(table.shape[2], device="cuda").expand(table.shape)
    touched = (column * c["page"] < lens) & (column >= (0 if s["from"] is None else s["from"][..., None] // c["page"]))
    page = table[touched].long()
    rows = (lens - column * c["page"]).clamp(max=c["page"])[touched]
    at = torch.arange(c["page"], device="cuda")
    x = _rows_plain(s, "k", page[:, None] * c["page"] + at)
    there = (at < rows[:, None])[..., None]
    high = x.masked_fill(~there, -math.inf).amax(1)
    low = x.masked_fill(~there, math.inf).amin(1)
    top = torch.maximum(high.abs(), low.abs()).amax(-1)
    scale = (top / torch.full_like(top, 127.0)).clamp(min=_LEAST)
    r = scale.reciprocal()[:, None]
    s["codes"][page, 0] = torch.ceil(high * r).clamp(-127.0, 127.0).to(torch.int8)
    s["codes"][page, 1] = torch.floor(low * r).clamp(-127.0, 127.0).to(torch.int8)
    s["page_scale"][page] = scale
    return s["codes"], s["page_scale"]


def _scores_plain(s):
    """Scores [nseq, Hkv, columns] of the pages: sums of whole numbers (exact in 32 bits), then two products."""
    c = s["case"]
    q = s["q"].float()
    top = q.abs().amax(-1)
    scale = (top / torch.full_like(top, 127.0)).clamp(min=_LEAST)
    code = (q * scale.reciprocal()[..., None]).round().clamp(-127.0, 127.0).view(c["nseq"], c["Hkv"], -1, c["dh"])
    page = s["table"].clamp(min=0).long()
    high, low = s["codes"][page, 0].float(), s["codes"][page, 1].float()
    total = code.clamp(min=0.0) @ high.transpose(-1, -2) + code.clamp(max=0.0) @ low.transpose(-1, -2)
    return (total * scale.view(c["nseq"], c["Hkv"], -1, 1) * s["page_scale"][page][:, :, None]).amax(2)


def _chosen_plain(s):
    """Numbers [nseq, Hkv, pages] of the chosen pages, ascending, and which of them exist: the first, the last, the best."""
    c = s["case"]
    score = _scores_plain(s)
    held = (s["lens"] + c["page"] - 1).div(c["page"], rounding_mode="floor")[..., None]
    column = torch.arange(score.shape[2], device="cuda")
    score = score.masked_fill((column == 0) | (column == held - 1), math.inf).masked_fill(column >= held, -math.inf)
    most = min(c["pages"], score.shape[2])
    best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :most]
    best = torch.sort(best, dim=-1).values
    return best, best < held


def _sparse_plain(s):
    c = s["case"]
    page, held = _chosen_plain(s)
    at = torch.arange(c["page"], device="cuda")
    row = page[..., None] * c["page"] + at
    there = (held[..., None] & (row < s["lens"][..., None, None])).flatten(2)
    slot = (s["table"].gather(2, page).clamp(min=0).long()[..., None] * c["page"] + at).flatten(2)
    return _attention_plain(s, _rows_plain(s, "k", slot), _rows_plain(s, "v", slot), there)


# ---- the library's calls -----------------------------------------------------------------------------------------
def _lib_handle():
    global _handle
    from paper_2502_03805_b200 import binding
    if _handle is None:
        _handle = binding.criticalkv_create(torch.cuda.current_device())
    return _handle


def _cache(s):
    if "cache" not in s:
        from paper_2502_03805_b200 import PagedCache
        c = s["case"]
        s["cache"] = PagedCache(Hq=c["Hq"], dtype=c["dtype"], format=_format(c), k_pages=s["k_pages"], v_pages=s["v_pages"],
                                k_scale=s["k_scale"], v_scale=s["v_scale"], k_group_scale=s["k_group"],
                                v_group_scale=s["v_group"], page_table=s["table"], handle=_lib_handle())
    return s["cache"]


def _append_own(s):
    c, cache = s["case"], _cache(s)
    if "rotary" not in s:
        from paper_2502_03805_b200 import Rotary
        s["rotary"] = Rotary(dh=c["dh"], frequencies=s["freq"], layout=c["layout"], handle=_lib_handle())
    q_out, lens = cache.append(s["q"], s["k"], s["v"], s["pos"], s["rotary"], s["start"], s["lens"], q_out=s["q_out"])
    if c["format"] == "plain":
        return q_out, s["k_pages"], s["v_pages"], lens
    return (q_out, *cache.load(lens, c["T"], align_right=True), lens)


def _store4_own(s):
    cache = _cache(s)
    cache.store(s["K"], s["V"], s["start"], s["lens"], idx=s["idx"], offsets=s["offsets"])
    return (*cache.load(s["lens"], s["columns"], align_right=not s["case"]["kept"]), s["lens"])


def _summary(s):
    if "summary" not in s:
        from paper_2502_03805_b200 import PageSummary
        s["summary"] = PageSummary(s["codes"], s["page_scale"])
    return s["summary"]


def run(state):
    s, op = state, state["case"]["op"]
    if op == "append":
        return _append_own(s) if own else _append_plain(s)
    if op == "store4":
        return _store4_own(s) if own else _store4_plain(s)
    if op == "attend4":
        return _cache(s).attend(s["q"], s["lens"]) if own else _attend4_plain(s)
    if op == "summarise":
        if own:
            _cache(s).summarise(_summary(s), s["lens"], s["from"])
            return s["codes"], s["page_scale"]
        return _summarise_plain(s)
    return _cache(s).attend_selected(s["q"], s["lens"], _summary(s), s["case"]["pages"]) if own else _sparse_plain(s)


def _held(c):
    """Bytes of a stored row."""
    size = 4 if c["dtype"] == "f32" else 2
    return {"plain": c["dh"] * size, "e4m3": c["dh"] + 4, "int8": c["dh"] + 4, "e2m1": c["dh"] * 9 // 16 + 4}[_format(c)]


def work(case):
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    counts = _counts(c)
    rows = sum(sum(row) for row in counts)
    held, page, dh = _held(c), c["page"], c["dh"]
    pages = sum(-(-x // page) for row in counts for x in row)
    heads = c["nseq"] * c["Hkv"]
    if c["op"] == "append":
        q = c["nseq"] * c["T"] * c["Hq"] * dh
        back = 0 if c["format"] == "plain" else 2 * rows * (held + dh * size)
        return {"bytes": 2 * q * size + 2 * rows * (dh * size + held) + back + c["nseq"] * c["T"] * 4 + c["rot"] * 4 + 4 * pages,
                "flops": 3 * c["nseq"] * c["T"] * (c["Hq"] + c["Hkv"]) * c["rot"]}
    if c["op"] == "store4":
        back = 2 * rows * (held + dh * size)
        return {"bytes": 2 * rows * (dh * size + held) + back + (4 * rows if c["kept"] else 0) + 8 * pages + 8 * heads,
                "flops": 8 * rows * dh}
    io = c["nseq"] * c["Hq"] * (2 * dh * size + 4)
    if c["op"] == "attend4":
        return {"bytes": 2 * rows * held + 4 * pages + io + 4 * heads, "flops": 4 * rows * dh * (c["Hq"] // c["Hkv"])}
    if c["op"] == "summarise":
        first = [[max(0, x - c["new"]) // page if c["new"] else 0 for x in row] for row in counts]
        touched = sum(-(-x // page) - f for row, at in zip(counts, first) for x, f in zip(row, at))
        rows = sum(x - f * page for row, at in zip(counts, first) for x, f in zip(row, at))
        return {"bytes": rows * held + touched * (2 * dh + 8) + 8 * heads, "flops": 2 * rows * dh}
    read = sum(min(x, c["pages"] * page) for row in counts for x in row)
    return {"bytes": pages * (2 * dh + 8) + 2 * read * held + io + 4 * heads,
            "flops": 4 * (pages + read) * dh * (c["Hq"] // c["Hkv"])}


# ---- 64 bits -----------------------------------------------------------------------------------------------------
def _exact_turn(s, x):
    c = s["case"]
    pairs = c["rot"] // 2
    angle = s["pos"].double()[..., None] * s["freq"]
    z = torch.polar(torch.ones_like(angle), angle)[:, None]
    y = x.double().contiguous()
    first, second = (slice(0, pairs), slice(pairs, 2 * pairs)) if c["layout"] == "half" else (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2))
    w = torch.complex(y[..., first], y[..., second]) * z
    y[..., first], y[..., second] = w.real, w.imag
    return y


def _nearest(y, bits, least, top):
    """Nearest value with `bits` fraction bits and exponents down to `least`, ties to even, at most `top`."""
    step = torch.exp2(torch.frexp(y.abs().clamp(min=2.0 ** least))[1].double() - (1.0 + bits))
    return (torch.round(y / step) * step).clamp(-top, top)


def _float32(x):
    """A result in 64 bits rounded as the definition of scales and codes has it: every operation a float32 one."""
    return x.float().double()


def _exact_held(c, x):
    """What rows stand for once they are stored."""
    x = x.double()
    if _format(c) == "plain":
        return x
    top = x.abs().amax(-1, keepdim=True)
    if _format(c) != "e2m1":
        scale = _float32(top / _TOP[_format(c)]).clamp(min=_LEAST)
        y = _float32(x * _float32(1.0 / scale))
        return (_nearest(y, 3, -6, 448.0) if _format(c) == "e4m3" else torch.round(y)) * scale
    scale = _float32(top / 2688.0).clamp(min=_LEAST)
    inverse = _float32(1.0 / scale)
    groups = x.unflatten(-1, (c["dh"] // 16, 16))
    sixth = float(np.float32(1) / np.float32(6))
    s = _nearest(_float32(_float32(groups.abs().amax(-1) * inverse) * sixth), 3, -6, 448.0)[..., None]
    factor = _float32(inverse[..., None] / s.clamp(min=2.0 ** -9))
    code = torch.where(s > 0, _nearest(_float32(groups * factor), 1, 0, 6.0), torch.zeros_like(groups))
    return (code * s).flatten(-2) * scale


def _exact_append(s):
    c = s["case"]
    dt = _DT[c["dtype"]]
    q = _exact_turn(s, s["q"])
    K, V = _exact_held(c, _exact_turn(s, s["k"]).to(dt)), _exact_held(c, s["v"])
    if c["format"] != "plain":
        return q, K, V, None
    outs = []
    for x, pages in ((_exact_turn(s, s["k"]), s["k_pages"]), (V, s["v_pages"])):
        out = torch.zeros(pages.shape, dtype=torch.float64, device="cuda")
        at = c["at"] + torch.arange(c["T"], device="cuda")
        for b in range(c["nseq"]):
            for h in range(c["Hkv"]):
                out[s["table"][b, h][at // c["page"]].long(), at % c["page"]] = x[b, h]
        outs.append(out)
    return q, outs[0], outs[1], None


def _exact_store4(s):
    c = s["case"]
    outs = []
    for x in (s["K"], s["V"]):
        out = torch.zeros((c["nseq"], c["Hkv"], s["columns"], c["dh"]), dtype=torch.float64, device="cuda")
        for b, row in enumerate(_counts(c)):
            done = 0
            for h, m in enumerate(row):
                part = x[b, h, :m] if s["idx"] is None else x[b, h, s["idx"][b, done:done + m].long()]
                done += m
                out[b, h, :m] = _exact_held(c, part)
        outs.append(out)
    return outs[0], outs[1], None


def _exact_rows(s, name, page, rows):
    """The rows of some pages of one head, `rows` in all, in 64 bits."""
    c, form = s["case"], _format(s["case"])
    pages = s[name + "_pages"][page]
    if form == "e2m1":
        low, high = (pages & 15).long(), (pages >> 4).long()
        x = torch.stack([low, high], -1).flatten(-2)
        size = x & 7
        y = torch.where(size < 2, size * 0.5, (1.0 + 0.5 * (size & 1).double()) * torch.exp2((size >> 1).double() - 1.0))
        y = torch.where(x > 7, -y, y).double() * s[name + "_group"][page].double().repeat_interleave(16, -1)
    else:
        y = pages.double()
    if form != "plain":
        y = y * s[name + "_scale"][page].double()[..., None]
    return y.reshape(-1, c["dh"])[:rows]


def _exact_heads(s, choose):
    """Attention of every head over the pages that choose(sequence, head, rows) names, the last of which may not be full."""
    c = s["case"]
    G = c["Hq"] // c["Hkv"]
    out = torch.zeros((c["nseq"], c["Hq"], c["dh"]), dtype=torch.float64, device="cuda")
    lse = torch.full((c["nseq"], c["Hq"]), -math.inf, dtype=torch.float64, device="cuda")
    for b, row in enumerate(_counts(c)):
        for h, m in enumerate(row):
            if m == 0:
                continue
            page = choose(b, h, m)
            rows = page.numel() * c["page"] - (-m) % c["page"]
            page = s["table"][b, h][page].long()
            K, V = _exact_rows(s, "k", page, rows), _exact_rows(s, "v", page, rows)
            logit = torch.matmul(K, s["q"][b, h * G:(h + 1) * G].double().T) / math.sqrt(c["dh"])
            lse[b, h * G:(h + 1) * G] = torch.logsumexp(logit, 0)
            out[b, h * G:(h + 1) * G] = torch.matmul(torch.softmax(logit, 0).T, V)
    return out, lse


def _exact_attend4(s):
    return _exact_heads(s, lambda b, h, m: torch.arange(-(-m // s["case"]["page"]), device="cuda"))


def _exact_sparse(s):
    """The choice goes by scores that are defined as products of a whole number with two float32 scales, each rounded."""
    c = s["case"]
    G = c["Hq"] // c["Hkv"]
    numbers = s["codes"].cpu().numpy().astype(np.int64)
    scales, table = s["page_scale"].cpu().numpy(), s["table"].cpu().numpy()
    queries = s["q"].float().cpu().numpy()

    def choose(b, h, m):
        held = -(-m // c["page"])
        x = queries[b, h * G:(h + 1) * G]
        scale = np.maximum(np.abs(x).max(1) / np.float32(127), np.float32(_LEAST))
        code = np.rint(x * (np.float32(1) / scale)[:, None]).astype(np.int64)
        up, down = numbers[table[b, h, :held], 0], numbers[table[b, h, :held], 1]
        total = np.maximum(code, 0) @ up.T + np.minimum(code, 0) @ down.T
        score = ((total.astype(np.float32) * scale[:, None]) * scales[table[b, h, :held]]).max(0)
        score[0] = score[held - 1] = np.inf
        best = np.lexsort((np.arange(held), -score))[:c["pages"]]
        return torch.from_numpy(np.sort(best)).cuda()

    return _exact_heads(s, choose)


def _exact_summarise(s):
    c = s["case"]
    out = torch.zeros_like(s["page_scale"], dtype=torch.float64)
    for b, row in enumerate(_counts(c)):
        for h, m in enumerate(row):
            column = torch.arange(max(0, m - c["new"]) // c["page"] if c["new"] else 0, -(-m // c["page"]), device="cuda")
            if column.numel():
                page = s["table"][b, h][column].long()
                x = _exact_rows(s, "k", page, page.numel() * c["page"]).view(-1, c["page"], c["dh"]).abs()
                x[-1, m - int(column[-1]) * c["page"]:] = 0.0
                out[page] = (x.amax((1, 2)) / 127.0).clamp(min=_LEAST)
    return None, out


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "store4": _exact_store4, "attend4": _exact_attend4, "summarise": _exact_summarise,
            "sparse": _exact_sparse}[case["op"]](s)
