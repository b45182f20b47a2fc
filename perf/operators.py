"""The paged-cache operators, as measurable cases: rows written into a paged
cache (a new token, the rows that a selection kept, whole prompts), cached rows
read back, and attention of a chunk of new tokens over the cached rows, from
one token of one sequence to a chunk of two thousand over a long prompt.

A cache is a pool of pages [n_pages, Hkv, page, d] for K and one for V, as
bf16, e4m3 or int8 (the 8-bit ones with one fp32 scale for each row), with a
table of the pages of every sequence; row t of sequence b lies in page
table[b, t // page] at t % page.  Rows are cached per KV head, so that their
number may differ between the heads of one sequence.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
CACHES = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
FLOATS = {"bf16": torch.bfloat16, "f32": torch.float32}

_WRITE = dict(op="write", kept=0, start=0, ragged="no", src="bf16", layout="heads", page=64, d=128)
_READ = dict(op="read", ragged="rows", out="bf16", page=64, d=128)
_ATTEND = dict(op="attend", ragged="rows", causal=True, layout="heads", page=64, d=128)


def listed():
    return [
        # the newest token of a decoding batch, behind the rows of its prompts
        dict(_WRITE, name="write_step_b32", B=32, Hkv=4, T=1, start=300, cache="e4m3", ragged="heads",
             layout="tokens"),
        # the rows kept by a selection over a batch of long prompts, another number for each head
        dict(_WRITE, name="write_kept_16k_b4", B=4, Hkv=4, T=16384, kept=256, cache="e4m3", ragged="heads"),
        # fp32 keys of short prompts of odd lengths, small pages
        dict(_WRITE, name="write_f32_1500_b3", B=3, Hkv=2, T=1500, d=64, cache="int8", src="f32", page=16,
             start=37, ragged="rows"),
        # two whole prompts of the longest kind as they are prefilled
        dict(_WRITE, name="write_prompt_32k_b2", B=2, Hkv=8, T=32768, cache="e4m3", layout="tokens"),
        # kept rows back in fp32 (to move a small cache elsewhere)
        dict(_READ, name="read_kept_b3", B=3, Hkv=2, T=701, d=64, cache="int8", out="f32", page=16, ragged="heads"),
        # the benchmark's prompts back as the keys and values that a selection scores and gathers
        dict(_READ, name="read_prompt_16k_b4", B=4, Hkv=4, T=16384, cache="e4m3"),
        # one decoding sequence over its kept rows: latency
        dict(_ATTEND, name="attend_step_kept", B=1, Hq=28, Hkv=4, T=321, n=1, cache="bf16", ragged="heads"),
        # a decoding batch over kept rows and the tokens since
        dict(_ATTEND, name="attend_step_kept_b32", B=32, Hq=28, Hkv=4, T=1100, n=1, cache="e4m3", ragged="heads"),
        # a decoding batch over whole prompts of a large model
        dict(_ATTEND, name="attend_step_32k_b16", B=16, Hq=64, Hkv=8, T=32768, n=1, cache="bf16"),
        # drafted tokens, another number for each sequence, of a small model with small pages
        dict(_ATTEND, name="attend_draft_b6", B=6, Hq=16, Hkv=2, T=5003, d=64, n=5, cache="int8", page=16,
             layout="tokens"),
        # the last chunk of a prompt as it is prefilled
        dict(_ATTEND, name="attend_chunk_8k", B=1, Hq=28, Hkv=4, T=8191, n=1024, cache="bf16", ragged="no",
             layout="tokens"),
        # a large chunk over a long prompt in 8 bits
        dict(_ATTEND, name="attend_chunk_32k", B=1, Hq=64, Hkv=8, T=32768, n=2048, cache="e4m3", ragged="no",
             layout="tokens"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = ((4, 1, 64), (16, 2, 64), (28, 4, 128), (28, 4, 128), (32, 8, 128), (32, 32, 128), (64, 8, 128), (8, 8, 64))


def draw(rng):
    op = rng.choice(("write", "read", "attend", "attend", "attend"))
    hq, hkv, d = rng.choice(HEADS)
    cache = rng.choice(("bf16", "e4m3", "e4m3", "int8"))
    page = rng.choice((16, 32, 64, 64, 128, 256))
    b = _log(rng, 1, 32)
    ragged = rng.choice(("no", "rows", "heads"))
    t = _log(rng, 1, 32768)
    while b * hkv * t * d > 1 << 26:               # values of K: those of the largest write
        b, t = (b + 1) // 2, t if b > 1 else t // 2 + 1
    layout = rng.choice(("heads", "tokens"))
    if op == "write":
        kept = rng.choice((0, 0, min(t, _log(rng, 1, 1024))))
        return dict(op=op, B=b, Hkv=hkv, T=t, d=d, kept=kept, start=rng.choice((0, rng.randint(1, 700))), page=page,
                    cache=cache, src=rng.choice(("bf16", "bf16", "f32")), ragged=ragged, layout=layout)
    if op == "read":
        return dict(op=op, B=b, Hkv=hkv, T=t, d=d, page=page, cache=cache, out=rng.choice(("bf16", "bf16", "f32")),
                    ragged=ragged)
    n = rng.choice((1, 1, rng.randint(2, 8), _log(rng, 9, 2048)))
    t = max(t, n)
    while b * hq * n * t > 1 << 31:                # half the logits of the largest chunk
        b, t = (b + 1) // 2, t if b > 1 else max(n, t // 2 + 1)
        if b == 1 and t == n:
            n = t = n // 2
    return dict(op=op, B=b, Hq=hq, Hkv=hkv, T=t, d=d, n=n, page=page, cache=cache, causal=rng.random() < 0.75,
                ragged=ragged, layout=layout)


# ---------------------------------------------------------------- sizes
def _counts(case, most, least=0, salt=0):
    """[B][Hkv] numbers of rows: `most` for the first sequence, fewer for some of the others (and their heads)."""
    rng = random.Random("%s %s %s" % (case["T"], case["B"], salt))
    got = []
    for b in range(case["B"]):
        n = most if b == 0 or case["ragged"] == "no" else max(least, most - rng.randint(0, most // 2 + 1))
        got.append([n if case["ragged"] != "heads" else max(least, n - rng.randint(0, n // 3))
                    for _ in range(case["Hkv"])])
    return got


def _new(case):
    """[B] new tokens of an attention case."""
    rng = random.Random("%s %s new" % (case["T"], case["B"]))
    return [case["n"] if b == 0 or case["ragged"] == "no" else rng.randint(min(1, case["n"]), case["n"])
            for b in range(case["B"])]


def _lens(case):
    """[B][Hkv] cached rows of a read or attention case; a chunk's own rows are among them."""
    return _counts(case, case["T"], case.get("n", 0))


def _rows(case):
    """[B][Hkv] rows that a write case writes."""
    return _counts(case, case["kept"] or case["T"], 1)


def _starts(case):
    """[B][Hkv] cached rows before a write."""
    return _counts(case, case["start"], 0, 1)


def _bytes(name):
    return {"bf16": 2, "f32": 4, "e4m3": 1, "int8": 1}[name]


def _row_bytes(case):
    """Bytes of one cached row of K and V with their scales."""
    return 2 * (case["d"] * _bytes(case["cache"]) + (0 if case["cache"] == "bf16" else 4))


def work(case):
    d = case["d"]
    if case["op"] == "write":
        rows = sum(map(sum, _rows(case)))
        return {"bytes": rows * (2 * d * _bytes(case["src"]) + _row_bytes(case) + (4 if case["kept"] else 0)),
                "flops": 4 * rows * d}
    rows = sum(map(sum, _lens(case)))
    if case["op"] == "read":
        whole = case["B"] * case["Hkv"] * case["T"]
        return {"bytes": rows * _row_bytes(case) + 2 * whole * d * _bytes(case["out"]), "flops": 2 * rows * d}
    gh, seen = case["Hq"] // case["Hkv"], 0
    for lens, n in zip(_lens(case), _new(case)):
        for length in lens:
            seen += sum(max(0, length - n + i + 1) if case["causal"] else length for i in range(n))
    return {"bytes": rows * _row_bytes(case) + 4 * case["B"] * case["Hq"] * case["n"] * d, "flops": 4 * d * gh * seen}


# ---------------------------------------------------------------- inputs
def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV)


def _int32(rows):
    return torch.tensor(rows, dtype=torch.int32, device=DEV)


def _tokens(x, layout):
    """[B, H, T, d] as given, or a view of a tensor whose tokens come first, as a projection leaves them."""
    return x.transpose(1, 2).contiguous().transpose(1, 2) if layout == "tokens" else x


def _keys(gen, b, hkv, t, d):
    """Keys with a few channels of large values, and values with a mean of their own in each channel."""
    k = _randn(gen, b, hkv, t, d)
    k += torch.where(torch.rand((1, hkv, 1, d), generator=gen, device=DEV) < 0.05, 4.0, 0.0)
    return k, _randn(gen, b, hkv, t, d).add_(_randn(gen, 1, hkv, 1, d), alpha=0.5)


def _quantise(x, cache):
    """Rows x [..., d] fp32 as a cache holds them: (values, scales or None)."""
    if cache == "bf16":
        return x.to(torch.bfloat16), None
    a = x.abs().amax(-1, keepdim=True)
    if cache == "e4m3":                            # the smallest power of two that brings the row within 448
        f, e = torch.frexp(a)
        e = (e - 9 + (f > 0.875)).clamp(min=-126)
        s = torch.ldexp(torch.ones_like(a), e)
        return (x * torch.ldexp(torch.ones_like(a), -e)).to(torch.float8_e4m3fn), s[..., 0]
    a = a.clamp(min=2.0 ** -100)
    most = torch.full_like(a, 127.0)
    return torch.round(x * (most / a)).to(torch.int8), (a / most)[..., 0]


def _pool(case, gen):
    """Pages in an order of their own for every sequence, a few of them unused."""
    rows = case["T"] if case["op"] != "write" else case["start"] + (case["kept"] or case["T"])
    per = -(-rows // case["page"])
    pages = case["B"] * per + 3
    order = torch.randperm(pages, generator=gen, device=DEV)[:case["B"] * per]
    shape = (pages, case["Hkv"], case["page"], case["d"])
    return shape, order.view(case["B"], per).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed((seed * 7919 + 31) & 0x7FFFFFFF)
    shape, table = _pool(case, gen)
    s = dict(case=case, table=table, k_scale=None, v_scale=None)
    if case["op"] == "write":
        k, v = _keys(gen, case["B"], case["Hkv"], case["T"], case["d"])
        s["k"], s["v"] = (_tokens(x.to(FLOATS[case["src"]]), case["layout"]) for x in (k, v))
        s["counts"], s["start"] = _int32(_rows(case)), _int32(_starts(case))
        s["idx"] = None
        if case["kept"]:                           # ascending tokens, -1 behind each head's number of them
            pick = torch.rand((case["B"], case["Hkv"], case["T"]), generator=gen, device=DEV).argsort(-1)
            pick = pick[..., :case["kept"]]
            last = torch.arange(case["kept"], device=DEV) >= s["counts"][..., None]
            pick = pick.masked_fill(last, case["T"]).sort(-1).values
            s["idx"] = torch.where(last, -1, pick).to(torch.int32)
        for name in ("k", "v"):
            s[name + "_pages"] = torch.ones(shape, device=DEV).to(CACHES[case["cache"]])
            if case["cache"] != "bf16":
                s[name + "_scale"] = torch.full(shape[:3], 0.5, device=DEV)
        return s
    for name, x in zip(("k", "v"), _keys(gen, *shape)):
        s[name + "_pages"], s[name + "_scale"] = _quantise(x, case["cache"])
    s["lens"] = _int32(_lens(case))
    if case["op"] == "attend":
        q = 1.5 * _randn(gen, case["B"], case["Hq"], case["n"], case["d"])
        s["q"] = _tokens(q.to(torch.bfloat16), case["layout"])
        s["new"] = _int32(_new(case))
    return s


# ---------------------------------------------------------------- plain forms
def _slots(s, rows):
    """Row numbers in a pool seen as [-1, d] of the cached rows `rows` [B, Hkv, n]."""
    case = s["case"]
    page = case["page"]
    at = torch.take_along_dim(s["table"].long()[:, None], rows // page, 2)
    head = torch.arange(case["Hkv"], device=DEV)[None, :, None]
    return (at * case["Hkv"] + head) * page + rows % page


def _raw(pages):
    return pages.view(torch.uint8) if pages.dtype == torch.float8_e4m3fn else pages


def _cached(s, name, dtype=torch.float32):
    """[B, Hkv, T, d] cached rows with their scales applied."""
    case = s["case"]
    rows = torch.arange(case["T"], device=DEV).expand(case["B"], case["Hkv"], -1)
    at = _slots(s, rows)
    pages = s[name + "_pages"]
    x = _raw(pages).view(-1, case["d"])[at].view(pages.dtype).to(dtype)
    scale = s[name + "_scale"]
    return x if scale is None else x * scale.view(-1)[at][..., None].to(dtype)


def _write(s):
    case = s["case"]
    most = case["kept"] or case["T"]
    row = torch.arange(most, device=DEV).expand(case["B"], case["Hkv"], -1)
    here = row < s["counts"][..., None]
    at = _slots(s, torch.where(here, row + s["start"][..., None], 0))[here]
    for name in ("k", "v"):
        x = s[name].float()
        if s["idx"] is not None:
            x = torch.take_along_dim(x, s["idx"].long().clamp(min=0)[..., None], 2)
        y, scale = _quantise(x, case["cache"])
        pages = _raw(s[name + "_pages"])
        pages.view(-1, case["d"])[at] = _raw(y)[here]
        if scale is not None:
            s[name + "_scale"].view(-1)[at] = scale[here]
    return {n: s[n] for n in ("k_pages", "v_pages", "k_scale", "v_scale")}


def _read(s):
    case = s["case"]
    past = torch.arange(case["T"], device=DEV) >= s["lens"][..., None]
    return {n: _cached(s, n).masked_fill_(past[..., None], 0.0).to(FLOATS[case["out"]]) for n in ("k", "v")}


def _hidden(s):
    """[B, Hkv, 1, n, T]: the keys that a query does not see."""
    case = s["case"]
    t = torch.arange(case["T"], device=DEV)
    i = torch.arange(case["n"], device=DEV)[:, None]
    lens, new = s["lens"][..., None, None], s["new"][:, None, None, None]
    seen = (t < lens) & (i < new)
    if case["causal"]:
        seen = seen & (t <= lens - new + i)
    return ~seen[:, :, None]


def _attend(s):
    case = s["case"]
    b, hkv, n, d, t = case["B"], case["Hkv"], case["n"], case["d"], case["T"]
    gh = case["Hq"] // hkv
    q = s["q"].float().reshape(b, hkv, gh * n, d) * (1.0 / math.sqrt(d))
    k = _cached(s, "k").transpose(2, 3).contiguous()
    p = (q @ k).view(b, hkv, gh, n, t).masked_fill_(_hidden(s), -math.inf)
    del k
    p -= p.amax(-1, keepdim=True).clamp(min=-3e38)
    p = p.exp_().view(b, hkv, gh * n, t)
    total = p.sum(-1, keepdim=True)
    o = (p @ _cached(s, "v")) / torch.where(total > 0, total, 1.0)
    return o.view(b, case["Hq"], n, d).to(torch.bfloat16)


def _own(s):
    import paper_2607_22586_amd as mm

    case = s["case"]
    cache = mm.PagedCache(s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["table"])
    if case["op"] == "write":
        mm.cache_write(cache, s["k"], s["v"], start=s["start"], counts=s["counts"], idx=s["idx"])
        return {n: s[n] for n in ("k_pages", "v_pages", "k_scale", "v_scale")}
    if case["op"] == "read":
        k, v = mm.cache_read(cache, s["lens"], case["T"], FLOATS[case["out"]])
        return {"k": k, "v": v}
    return mm.chunk_attention(s["q"], cache, s["lens"], q_counts=s["new"], T=case["T"], causal=case["causal"])


def run(state):
    if own:
        return _own(state)
    return {"write": _write, "read": _read, "attend": _attend}[state["case"]["op"]](state)


# ---------------------------------------------------------------- in 64 bits
def _e4m3(x):
    """x rounded to the nearest e4m3 value (three bits behind the first, down to 2^-9), ties to even."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def _exact_write(s):
    case = s["case"]
    got = {n: None for n in ("k_pages", "v_pages", "k_scale", "v_scale")}
    counts, start, table = s["counts"].tolist(), s["start"].tolist(), s["table"].long()
    for name in ("k", "v"):
        x = s[name].double()
        a = x.abs().amax(-1)
        if case["cache"] == "e4m3":
            scale = torch.exp2(torch.ceil(torch.log2(a / 448.0)).clamp(min=-126))
            x = _e4m3(x / scale[..., None])
        elif case["cache"] == "int8":
            scale = a / 127.0
        pages = s[name + "_pages"].double()
        scales = None if s[name + "_scale"] is None else s[name + "_scale"].double()
        for b in range(case["B"]):
            for c in range(case["Hkv"]):
                n, first = counts[b][c], start[b][c]
                at = torch.arange(first, first + n, device=DEV)
                pick = torch.arange(n, device=DEV) if s["idx"] is None else s["idx"][b, c, :n].long()
                pages[table[b, at // case["page"]], c, at % case["page"]] = x[b, c, pick]
                if scales is not None:
                    scales[table[b, at // case["page"]], c, at % case["page"]] = scale[b, c, pick]
        got[name + "_pages"] = None if case["cache"] == "int8" else pages   # whole numbers
        got[name + "_scale"] = scales
    return got


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "write":
        return _exact_write(s)
    lens = s["lens"].tolist()
    got = {"k": [], "v": []}
    for b in range(case["B"]):
        for c in range(case["Hkv"]):
            for name in ("k", "v"):
                x = s[name + "_pages"][s["table"][b].long(), c] if case["cache"] != "e4m3" else \
                    s[name + "_pages"].view(torch.uint8)[s["table"][b].long(), c].view(torch.float8_e4m3fn)
                x = x.double()
                if s[name + "_scale"] is not None:
                    x = x * s[name + "_scale"][s["table"][b].long(), c].double()[..., None]
                x = x.reshape(-1, case["d"])[:case["T"]].clone()
                x[lens[b][c]:] = 0.0
                got[name].append(x)
    if case["op"] == "read":
        return {n: torch.stack(x).view(case["B"], case["Hkv"], case["T"], case["d"]) for n, x in got.items()}
    new, gh = s["new"].tolist(), case["Hq"] // case["Hkv"]
    out = torch.zeros((case["B"], case["Hq"], case["n"], case["d"]), dtype=torch.float64, device=DEV)
    for b in range(case["B"]):
        for h in range(case["Hq"]):
            c = h // gh
            length, n = lens[b][c], new[b]
            k, v = (got[name][b * case["Hkv"] + c][:length] for name in ("k", "v"))
            score = s["q"][b, h, :n].double() @ k.t().contiguous() / math.sqrt(case["d"])
            if case["causal"]:
                last = length - n + torch.arange(n, device=DEV)[:, None]
                score.masked_fill_(torch.arange(length, device=DEV) > last, -math.inf)
            if length:
                out[b, h, :n] = torch.nan_to_num(torch.softmax(score, -1)) @ v
    return out
