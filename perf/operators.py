"""Decoding on a compressed cache, operator by operator: what is measured, and the plain form of each.

Four operators that follow the compression step in a serving loop:

  rope    rotary positions of the new tokens' queries and keys
  store   rows written into a paged cache (new tokens, or the rows a selection kept), quantised to 8 bits a value
  load    rows of a paged cache read back into a dense tensor
  decode  attention of one new token over the paged cache, every KV head with its own length

A case is a dict of plain values; prepare() makes its inputs on the GPU from a seed, run() makes one pass.  With
`own` false run() computes the operators with elementary torch operations in 32 bits (angles in 64); with `own` true
it calls the library.
"""
import math
import random

import numpy as np
import torch

own = False
_handle = None       # the library handle a program keeps for its lifetime

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_TOP = {"e4m3": 448.0, "int8": 127.0}
_CODE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
_LEAST = 2.0 ** -100     # smallest scale of a stored row


# ---- cases -------------------------------------------------------------------------------------------------------
def listed():
    head = dict(Hq=32, Hkv=8, dh=128, dtype="bf16")          # 32 query heads on 8 KV heads, as the 32-layer workload
    return [
        # one new token of one sequence, far into a long context
        dict(name="rope one token", op="rope", nseq=1, T=1, rot=128, layout="half", scaling="none", at=131000, **head),
        # one new token of each of 61 sequences; only half of a 64-wide head is rotated, pairs interleaved, float32
        dict(name="rope 61 tokens, part of head", op="rope", nseq=61, T=1, Hq=8, Hkv=2, dh=64, dtype="f32", rot=32,
             layout="interleaved", scaling="linear", at=5000),
        # a whole prompt of the headline length, frequencies scaled for the long context
        dict(name="rope prompt 32768", op="rope", nseq=1, T=32768, rot=128, layout="half", scaling="banded", at=0, **head),
        # the new tokens of 16 sequences appended to their caches
        dict(name="store 16 tokens e4m3", op="store", nseq=16, n=1, kept=0, page=64, format="e4m3", at=6553, **head),
        # the rows an adaptive selection kept (20 % of 32768 per head on average), 8 layers at once
        dict(name="store kept rows e4m3", op="store", nseq=8, n=32768, kept=6553, page=64, format="e4m3", at=0, **head),
        # prompt chunks of three sequences, float32 model, odd length, behind rows already there
        dict(name="store 3 chunks int8", op="store", nseq=3, n=4099, kept=0, page=16, format="int8", at=77, Hq=4, Hkv=4,
             dh=64, dtype="f32"),
        # a small ragged cache read back for another compression step
        dict(name="load short int8", op="load", nseq=2, rows=409, spread=0.5, page=16, format="int8", Hq=8, Hkv=2, dh=64,
             dtype="f32"),
        # the kept rows of 8 layers read back
        dict(name="load kept rows e4m3", op="load", nseq=8, rows=6553, spread=0.8, page=64, format="e4m3", **head),
        # one sequence, a short cache: latency
        dict(name="decode one, 819 rows", op="decode", nseq=1, rows=819, spread=0.5, page=64, format="plain", **head),
        # 32 sequences on caches an adaptive budget compressed to 20 % of 32768, 8 bits a value
        dict(name="decode 32, kept rows e4m3", op="decode", nseq=32, rows=6553, spread=0.8, page=64, format="e4m3", **head),
        # float32 model with a 64-wide head, a few sequences, odd lengths, one head empty
        dict(name="decode 5, float32 int8", op="decode", nseq=5, rows=1237, spread=1.0, page=16, format="int8", Hq=8,
             Hkv=2, dh=64, dtype="f32"),
        # two uncompressed caches of 131072 rows, 40 query heads on 8 KV heads
        dict(name="decode 2, 131072 rows", op="decode", nseq=2, rows=131072, spread=0.0, page=128, format="plain", Hq=40,
             Hkv=8, dh=128, dtype="bf16"),
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
    op = rng.choice(["rope", "store", "load", "decode", "decode"])
    Hkv = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 4, 5, 8])
    dh = rng.choice([64, 128])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    c = dict(op=op, Hq=Hkv * G, Hkv=Hkv, dh=dh, dtype=dtype)
    if op == "rope":
        T = _log(rng, 1, 32768)
        nseq = _log(rng, 1, max(1, min(64, 32768 // T)))
        return dict(c, nseq=nseq, T=T, rot=rng.choice([dh, dh // 2, dh // 4]), layout=rng.choice(["half", "interleaved"]),
                    scaling=rng.choice(["none", "linear", "banded"]), at=rng.randrange(131072 - T + 1))
    c.update(page=rng.choice([16, 32, 64, 128]), format=rng.choice(["plain", "e4m3", "int8"]))
    if op == "store":
        n = _log(rng, 1, 32768)
        nseq = _log(rng, 1, max(1, min(64, 131072 // n)))
        kept = rng.choice([0, max(1, n // 5)]) if n >= 8 else 0
        return dict(c, nseq=nseq, n=n, kept=kept, at=rng.randrange(200))
    rows = _log(rng, 16, 65536)
    nseq = _log(rng, 1, max(1, min(64, (65536 if op == "load" else 131072) // rows)))
    return dict(c, nseq=nseq, rows=rows, spread=rng.choice([0.0, 0.5, 0.8, 1.0]))


def _ragged(nseq, Hkv, mean, spread, most):
    """Row counts [nseq][Hkv] of the heads, the same for every seed; with spread 1 the last head is empty."""
    r = random.Random("%d %d %d %r" % (nseq, Hkv, mean, spread))
    at = [[max(0, min(most, round(mean * (1 + spread * r.uniform(-1, 1))))) for _ in range(Hkv)] for _ in range(nseq)]
    if spread >= 1.0:
        at[-1][-1] = 0
    return at


def _counts(c):
    """Rows of every head of a case: stored by `store`, held for `load` and `decode`."""
    if c["op"] == "store":
        if not c["kept"]:
            return [[c["n"]] * c["Hkv"] for _ in range(c["nseq"])]
        return _ragged(c["nseq"], c["Hkv"], c["kept"], 0.8, c["n"])
    return _ragged(c["nseq"], c["Hkv"], c["rows"], c["spread"], 2 * c["rows"])


# ---- inputs ------------------------------------------------------------------------------------------------------
def _frequencies(c):
    """Radians a position for each pair of the rotated part, in 64 bits.  linear: positions four times denser; banded:
    wavelengths above 8192 positions eight times slower, below 2048 as they were, a linear blend between."""
    i = np.arange(c["rot"] // 2, dtype=np.float64)
    f = 500000.0 ** (-2.0 * i / c["rot"])
    if c["scaling"] == "linear":
        f = f / 4.0
    elif c["scaling"] == "banded":
        wave = 2.0 * np.pi / f
        keep = np.clip((8192.0 / wave - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        f = (1.0 - keep) * f / 8.0 + keep * f
    return f


def _factor(c):
    return 1.125 if c["scaling"] == "linear" else 1.0


def _rows_like_cache(g, shape, dtype, keys):
    """Rows as a cache holds them: keys with a few large channels, values whose norm varies from token to token."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    if keys:
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
    dt = _DT[c["dtype"]]
    s = dict(case=c)
    if c["op"] == "rope":
        both = torch.randn((c["nseq"], c["T"], c["Hq"] + 2 * c["Hkv"], c["dh"]), generator=g, device="cuda").to(dt)
        q, k = both[:, :, :c["Hq"]], both[:, :, c["Hq"]:c["Hq"] + c["Hkv"]]      # parts of one projection's output
        s.update(both=both, q=q.transpose(1, 2), k=k.transpose(1, 2))
        first = torch.randint(0, 64, (c["nseq"], 1), generator=g, device="cuda", dtype=torch.int32)
        s["pos"] = (c["at"] + first + torch.arange(c["T"], device="cuda", dtype=torch.int32)).contiguous()
        s["freq"] = torch.from_numpy(_frequencies(c)).cuda()
        s["q_out"] = torch.empty((c["nseq"], c["Hq"], c["T"], c["dh"]), dtype=dt, device="cuda")
        s["k_out"] = torch.empty((c["nseq"], c["Hkv"], c["T"], c["dh"]), dtype=dt, device="cuda")
        return s
    counts = _counts(c)
    at = c.get("at", 0)
    s["table"], pages = _table(c, [[x + at for x in row] for row in counts], g)
    code = _CODE.get(c["format"], dt)
    pool = (pages, c["page"], c["dh"])
    counts_t = torch.tensor(counts, dtype=torch.int32, device="cuda")
    if c["op"] == "store":
        s["k_pages"], s["v_pages"] = (torch.zeros(pool, device="cuda").to(code) for _ in range(2))
        s["k_scale"], s["v_scale"] = (torch.zeros(pool[:2], device="cuda") if c["format"] != "plain" else None for _ in range(2))
        src = (c["nseq"], c["Hkv"], c["n"], c["dh"])
        s["K"], s["V"] = _rows_like_cache(g, src, dt, True), _rows_like_cache(g, src, dt, False)
        s["start"] = torch.full((c["nseq"], c["Hkv"]), at, dtype=torch.int32, device="cuda")
        s["lens"] = torch.zeros_like(s["start"])
        s["idx"] = s["offsets"] = None
        if c["kept"]:
            order = torch.rand(src[:3], generator=g, device="cuda").argsort(-1).argsort(-1)
            s["idx"] = (order < counts_t[..., None]).nonzero()[:, 2].to(torch.int32)
            total = counts_t.sum(1)
            most = int(total.max())
            idx = torch.full((c["nseq"], most), -1, dtype=torch.int32, device="cuda")
            idx[torch.arange(most, device="cuda") < total[:, None]] = s["idx"]
            s["idx"] = idx
            s["offsets"] = torch.nn.functional.pad(counts_t.cumsum(1), (1, 0)).to(torch.int32)
            s["total"] = [sum(row) for row in counts]
        return s
    s["lens"] = counts_t
    s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"] = None, None, None, None
    for name in ("k", "v"):
        x = _rows_like_cache(g, pool, dt, name == "k")
        if c["format"] != "plain":
            x = x.float()
            scale = x.abs().amax(-1).div(_TOP[c["format"]]).clamp(min=_LEAST)
            s[name + "_scale"] = scale
            x = x / scale[..., None]
            x = x.clamp(-448.0, 448.0).to(code) if c["format"] == "e4m3" else x.round().clamp(-127, 127).to(code)
        s[name + "_pages"] = x
    s["columns"] = max(1, max(max(row) for row in counts))
    if c["op"] == "load":
        out = (c["nseq"], c["Hkv"], s["columns"], c["dh"])
        s["K_out"], s["V_out"] = torch.zeros(out, dtype=dt, device="cuda"), torch.zeros(out, dtype=dt, device="cuda")
    else:
        # queries whose logits have a standard deviation near 2.5 over these keys
        s["q"] = (torch.randn((c["nseq"], c["Hq"], c["dh"]), generator=g, device="cuda") * (2.5 / math.sqrt(3.0))).to(dt)
    return s


# ---- plain forms -------------------------------------------------------------------------------------------------
def _rope_plain(s):
    c, h = s["case"], s["case"]["rot"] // 2
    angle = s["pos"].double()[:, None, :, None] * s["freq"]
    cos, sin = (angle.cos() * _factor(c)).float(), (angle.sin() * _factor(c)).float()

    def turn(x):
        y = x.float()
        if c["layout"] == "half":
            a, b = y[..., :h], y[..., h:2 * h]
            y = torch.cat([a * cos - b * sin, b * cos + a * sin, y[..., 2 * h:]], -1)
        else:
            a, b = y[..., 0:2 * h:2], y[..., 1:2 * h:2]
            z = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
            y = torch.cat([z, y[..., 2 * h:]], -1)
        return y.to(x.dtype)

    return turn(s["q"]), turn(s["k"])


def _quantise_plain(x, form):
    """Codes and scales of rows: scale = largest magnitude / largest code, code = value * (1 / scale) rounded."""
    y = x.float()
    top = y.abs().amax(-1)
    scale = (top / torch.full_like(top, _TOP[form])).clamp(min=_LEAST)
    y = y * scale.reciprocal()[..., None]
    if form == "e4m3":
        return y.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8), scale
    return y.round().clamp(-127.0, 127.0).to(torch.int8), scale


def _slots(table, page, seq, head, row):
    return table[seq, head, row // page].long() * page + row % page


def _store_plain(s):
    c = s["case"]
    if s["idx"] is None:
        row = torch.arange(c["n"], device="cuda").expand(c["nseq"], c["Hkv"], c["n"])
        seq = torch.arange(c["nseq"], device="cuda")[:, None, None].expand_as(row)
        head = torch.arange(c["Hkv"], device="cuda")[None, :, None].expand_as(row)
        src = row
    else:
        counts = s["offsets"].diff(dim=1)
        flat = torch.repeat_interleave(torch.arange(counts.numel(), device="cuda"), counts.flatten(),
                                       output_size=sum(s["total"]))
        seq, head = flat // c["Hkv"], flat % c["Hkv"]
        before = torch.nn.functional.pad(counts.flatten().cumsum(0), (1, 0))
        row = torch.arange(sum(s["total"]), device="cuda") - before[flat]
        src = s["idx"][seq, s["offsets"][seq, head] + row].long()
    to = _slots(s["table"], c["page"], seq, head, row + s["start"][seq, head])
    for name in ("k", "v"):
        x = s[name.upper()][seq, head, src]
        pages = s[name + "_pages"]
        if c["format"] == "plain":
            pages.view(-1, c["dh"])[to] = x
            continue
        code, scale = _quantise_plain(x, c["format"])
        pages.view(code.dtype).view(-1, c["dh"])[to] = code
        s[name + "_scale"].view(-1)[to] = scale
    s["lens"].copy_(s["start"] + (c["n"] if s["idx"] is None else s["offsets"].diff(dim=1)))


def _gather_plain(s, name, n):
    """Rows 0..n-1 of every head as float32 [nseq, Hkv, n, dh]; rows behind a head's length are of any page."""
    c, table = s["case"], s["table"]
    row = torch.arange(n, device="cuda")
    slot = table[:, :, row // c["page"]].clamp(min=0).long() * c["page"] + row % c["page"]
    pages = s[name + "_pages"]
    if c["format"] == "e4m3":
        x = pages.view(torch.uint8).view(-1, c["dh"])[slot].view(torch.float8_e4m3fn).float()
    else:
        x = pages.view(-1, c["dh"])[slot].float()
    return x if c["format"] == "plain" else x * s[name + "_scale"].view(-1)[slot][..., None]


def _load_plain(s):
    n = s["columns"]
    there = (torch.arange(n, device="cuda") < s["lens"][..., None])[..., None]
    for name, out in (("k", s["K_out"]), ("v", s["V_out"])):
        out.copy_(torch.where(there, _gather_plain(s, name, n).to(out.dtype), out))


def _decode_plain(s):
    c, n = s["case"], s["columns"]
    q = s["q"].float().view(c["nseq"], c["Hkv"], -1, c["dh"])
    logit = q @ _gather_plain(s, "k", n).transpose(-1, -2) * (1.0 / math.sqrt(c["dh"]))
    there = torch.arange(n, device="cuda") < s["lens"][..., None, None]
    logit = logit.masked_fill(~there, -math.inf)
    top = logit.amax(-1, keepdim=True)
    none = (s["lens"] == 0)[..., None, None]
    w = torch.exp(logit - top.masked_fill(none, 0.0))
    total = w.sum(-1, keepdim=True)
    v = _gather_plain(s, "v", n).masked_fill(~there.transpose(-1, -2), 0.0)
    out = (w @ v / total).masked_fill(none, 0.0)
    lse = (top + torch.log(total)).masked_fill(none, -math.inf)
    return out.to(s["q"].dtype).view(c["nseq"], c["Hq"], c["dh"]), lse.view(c["nseq"], c["Hq"])


# ---- the library's calls -----------------------------------------------------------------------------------------
def _lib_handle():
    global _handle
    from paper_2502_03805_b200 import binding
    if _handle is None:
        _handle = binding.criticalkv_create(torch.cuda.current_device())
    return _handle


def _rope_own(s):
    c = s["case"]
    if "rotary" not in s:
        from paper_2502_03805_b200 import Rotary
        s["rotary"] = Rotary(dh=c["dh"], frequencies=s["freq"], layout=c["layout"], factor=_factor(c), handle=_lib_handle())
    return s["rotary"].rotate(s["q"], s["k"], s["pos"], q_out=s["q_out"], k_out=s["k_out"])


def _cache(s):
    if "cache" not in s:
        from paper_2502_03805_b200 import PagedCache
        c = s["case"]
        s["cache"] = PagedCache(Hq=c["Hq"], dtype=c["dtype"], format=c["format"], k_pages=s["k_pages"],
                                v_pages=s["v_pages"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                                page_table=s["table"], handle=_lib_handle())
    return s["cache"]


def _state(s):
    return {n: s[n] for n in ("k_pages", "v_pages", "k_scale", "v_scale", "lens")}


def run(state):
    s, op = state, state["case"]["op"]
    if op == "rope":
        return _rope_own(s) if own else _rope_plain(s)
    if op == "store":
        if own:
            _cache(s).store(s["K"], s["V"], start=s["start"], lens_out=s["lens"], idx=s["idx"], offsets=s["offsets"])
        else:
            _store_plain(s)
        return _state(s)
    if op == "load":
        if own:
            _cache(s).load(s["lens"], K_out=s["K_out"], V_out=s["V_out"])
        else:
            _load_plain(s)
        return s["K_out"], s["V_out"]
    return _cache(s).attend(s["q"], s["lens"]) if own else _decode_plain(s)


def work(case):
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "rope":
        rows = c["nseq"] * c["T"] * (c["Hq"] + c["Hkv"])
        return {"bytes": 2 * rows * c["dh"] * size + c["nseq"] * c["T"] * 4 + c["rot"] * 4, "flops": rows * c["rot"] * 3}
    rows = sum(sum(row) for row in _counts(c))
    held = c["dh"] * size if c["format"] == "plain" else c["dh"] + 4      # bytes of a stored row
    pages = 4 * sum(-(-x // c["page"]) for row in _counts(c) for x in row)
    if c["op"] in ("store", "load"):
        index = rows * 4 if c["op"] == "store" and c["kept"] else 0
        return {"bytes": 2 * rows * (c["dh"] * size + held) + index + pages + 8 * c["nseq"] * c["Hkv"],
                "flops": 2 * rows * c["dh"] * (0 if c["format"] == "plain" else 2)}
    io = c["nseq"] * c["Hq"] * (2 * c["dh"] * size + 4)
    return {"bytes": 2 * rows * held + pages + io + 4 * c["nseq"] * c["Hkv"],
            "flops": 4 * rows * c["dh"] * (c["Hq"] // c["Hkv"])}


# ---- 64 bits -----------------------------------------------------------------------------------------------------
def _exact_rope(s):
    c = s["case"]
    pairs = c["rot"] // 2
    z = torch.polar(torch.full((1,), _factor(c), dtype=torch.float64, device="cuda").expand(c["nseq"], c["T"], pairs).contiguous(),
                    s["pos"].double()[..., None] * s["freq"])
    outs = []
    for x in (s["q"], s["k"]):
        y = x.double().contiguous()
        if c["layout"] == "half":
            first, second = slice(0, pairs), slice(pairs, 2 * pairs)
        else:
            first, second = slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)
        w = torch.complex(y[..., first], y[..., second]) * z[:, None]
        y[..., first], y[..., second] = w.real, w.imag
        outs.append(y)
    return tuple(outs)


def _exact_e4m3(y):
    """Nearest value with 3 fraction bits and exponents down to -6, ties to even, at most 448."""
    step = torch.exp2(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1].double() - 4.0)
    return (torch.round(y / step) * step).clamp(-448.0, 448.0)


def _exact_store(s):
    c = s["case"]
    out = {"lens": None}
    counts = _counts(c)
    for name in ("k", "v"):
        pages = torch.zeros(s[name + "_pages"].shape, dtype=torch.float64, device="cuda")
        scales = torch.zeros(pages.shape[:2], dtype=torch.float64, device="cuda")
        for b in range(c["nseq"]):
            done = 0
            for h in range(c["Hkv"]):
                m = counts[b][h]
                x = s[name.upper()][b, h]
                if s["idx"] is not None:
                    x = x[s["idx"][b, done:done + m].long()]
                    done += m
                x = x.double()
                at = c["at"] + torch.arange(m, device="cuda")
                page, slot = s["table"][b, h][torch.div(at, c["page"], rounding_mode="floor")].long(), at % c["page"]
                if c["format"] == "plain":
                    pages[page, slot] = x
                    continue
                scale = torch.clamp(x.abs().max(-1).values / _TOP[c["format"]], min=_LEAST)
                y = x / scale[:, None]
                pages[page, slot] = _exact_e4m3(y) if c["format"] == "e4m3" else torch.round(y)
                scales[page, slot] = scale
        out[name + "_pages"] = None if c["format"] == "int8" else pages      # codes of int8 are whole numbers
        out[name + "_scale"] = None if c["format"] == "plain" else scales
    return out


def _exact_rows(s, name, b, h, m):
    c = s["case"]
    at = torch.arange(m, device="cuda")
    page, slot = s["table"][b, h][torch.div(at, c["page"], rounding_mode="floor")].long(), at % c["page"]
    pages = s[name + "_pages"]
    x = (pages.view(torch.uint8)[page, slot].view(pages.dtype) if c["format"] == "e4m3" else pages[page, slot]).double()
    return x if c["format"] == "plain" else x * s[name + "_scale"][page, slot].double()[:, None]


def _exact_load(s):
    c = s["case"]
    outs = []
    for name, like in (("k", s["K_out"]), ("v", s["V_out"])):
        out = torch.zeros(like.shape, dtype=torch.float64, device="cuda")
        for b, row in enumerate(_counts(c)):
            for h, m in enumerate(row):
                out[b, h, :m] = _exact_rows(s, name, b, h, m)
        outs.append(out)
    return tuple(outs)


def _exact_decode(s):
    c = s["case"]
    G = c["Hq"] // c["Hkv"]
    out = torch.zeros((c["nseq"], c["Hq"], c["dh"]), dtype=torch.float64, device="cuda")
    lse = torch.full((c["nseq"], c["Hq"]), -math.inf, dtype=torch.float64, device="cuda")
    for b, row in enumerate(_counts(c)):
        for h, m in enumerate(row):
            if m == 0:
                continue
            K, V = _exact_rows(s, "k", b, h, m), _exact_rows(s, "v", b, h, m)
            logit = torch.matmul(K, s["q"][b, h * G:(h + 1) * G].double().T) / math.sqrt(c["dh"])
            lse[b, h * G:(h + 1) * G] = torch.logsumexp(logit, 0)
            out[b, h * G:(h + 1) * G] = torch.matmul(torch.softmax(logit, 0).T, V)
    return out, lse


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "store": _exact_store, "load": _exact_load, "decode": _exact_decode}[case["op"]](s)
