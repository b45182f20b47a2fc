"""A prompt that is answered several times, as measurable cases: attention of
whole prompts over themselves (a batch, or sequences of different lengths packed
one behind the other), the pages of a cache held, forked and compacted, and
attention of a batch whose sequences share a long prefix, read once for all.

A cache is a pool of pages [n_pages, Hkv, page, d] for K and one for V, as bf16,
e4m3 or int8 (the 8-bit ones with one fp32 scale for each row), with a table of
the pages of every sequence and the number of table entries that name each page
(0: free).  Row t of sequence b lies in page table[b, t // page] at t % page.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
CACHES = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}

_PROMPT = dict(op="prompt", S=0, causal=True, lse=False, layout="tokens", d=128)
_HOLD = dict(op="hold", Hkv=4, d=128, page=64, cache="e4m3", ragged="heads")
_FORK = dict(op="fork", page=64, d=128, ragged="heads")
_COMPACT = dict(op="compact", page=64, d=128, ragged="heads")
_SHARED = dict(op="shared", ragged="heads", causal=True, layout="heads", page=64, d=128, n=1)


def listed():
    return [
        # questions of a few words to a few hundred, packed, of a small model
        dict(_PROMPT, name="prompt_packed_3k", B=1, Hq=16, Hkv=2, T=3001, S=23, d=64),
        # images of different sizes: every patch sees its image's patches
        dict(_PROMPT, name="prompt_images_8k", B=1, Hq=16, Hkv=16, T=8190, S=7, d=64, causal=False, lse=True),
        # the benchmark's batch of prompts as they are prefilled
        dict(_PROMPT, name="prompt_16k_b4", B=4, Hq=28, Hkv=4, T=16384),
        # a decoding batch before its next tokens: a few sequences need a page, one has ended
        dict(_HOLD, name="hold_step_b32", B=32, T=700, n_pages=600, max_pages=24),
        # a full server: many long sequences, some ended, some new
        dict(_HOLD, name="hold_server_b256", B=256, Hkv=1, d=64, T=16384, n_pages=65521, max_pages=512),
        # four answers to one prompt of kept rows: latency
        dict(_FORK, name="fork_kept_b4", B=4, Hkv=4, T=321, cache="bf16", each=4),
        # eight answers to each of eight prompts whose heads kept different numbers of rows
        dict(_FORK, name="fork_b64", B=64, Hkv=8, T=5003, cache="e4m3", each=8),
        # the rows that a second selection kept of small caches with small pages
        dict(_COMPACT, name="compact_kept_b3", B=3, Hkv=2, T=1500, d=64, cache="int8", page=16, kept=256),
        # a quarter of each head's rows of eight long prompts
        dict(_COMPACT, name="compact_32k_b8", B=8, Hkv=8, T=32768, cache="bf16", kept=8192),
        # two prompts' kept rows with four answers each: latency
        dict(_SHARED, name="shared_kept_b8", B=8, G=2, Hq=28, Hkv=4, T=512, own=70, cache="bf16"),
        # drafted tokens of answers to one odd prompt of a small model, small pages
        dict(_SHARED, name="shared_draft_b15", B=15, G=1, Hq=16, Hkv=2, T=5003, own=333, n=4, d=64, cache="int8",
             page=16, layout="tokens"),
        # many answers to two of the longest prompts of a large model
        dict(_SHARED, name="shared_32k_b64", B=64, G=2, Hq=64, Hkv=8, T=32768, own=600, cache="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = ((4, 1, 64), (16, 2, 64), (28, 4, 128), (28, 4, 128), (32, 8, 128), (32, 32, 128), (64, 8, 128), (8, 8, 64))


def draw(rng):
    op = rng.choice(("prompt", "prompt", "shared", "shared", "shared", "hold", "fork", "compact"))
    hq, hkv, d = rng.choice(HEADS)
    layout = rng.choice(("heads", "tokens"))
    if op == "prompt":
        b, t, s = _log(rng, 1, 8), _log(rng, 1, 16384), 0
        if rng.random() < 0.5:
            b, s = 1, _log(rng, 1, 64)
        while b * hq * t * t * d > 4 * 28 * 128 * 16384 ** 2:
            b, t = (b + 1) // 2, t if b > 1 else t // 2 + 1
        return dict(op=op, B=b, Hq=hq, Hkv=hkv, T=t, S=s, d=d, causal=rng.random() < 0.75, lse=rng.random() < 0.3,
                    layout=layout)
    cache = rng.choice(("bf16", "e4m3", "e4m3", "int8"))
    page = rng.choice((16, 32, 64, 64, 128, 256))
    ragged = rng.choice(("no", "rows", "heads"))
    base = dict(op=op, Hkv=hkv, d=d, page=page, cache=cache, ragged=ragged)
    if op == "shared":
        g = rng.choice((1, 1, 2, rng.randint(2, 6)))
        b, n = g * _log(rng, 1, 32), rng.choice((1, 1, 1, rng.randint(2, 8)))
        t, mine = _log(rng, 1, 32768), n + _log(rng, 1, 1000)
        while b * hkv * (t + mine) * d > 1 << 31 or b * hq * n * (t + mine) > 1 << 28:
            t = t // 2 + 1
        return dict(base, B=b, G=g, Hq=hq, T=t, own=mine, n=n, causal=rng.random() < 0.75, layout=layout)
    if op == "hold":
        t, b = _log(rng, 1, 16384), _log(rng, 1, 256)
        most = -(-t // page) + rng.randint(1, 9)
        n = max(1, min(65521, int(b * -(-t // page) * rng.uniform(0.8, 1.6))))
        while n * hkv * page * d > 1 << 30:
            n = n // 2 + 1
        return dict(base, B=b, T=t, n_pages=n, max_pages=most)
    t = _log(rng, 1, 32768)
    if op == "fork":
        each = _log(rng, 2, 16)
        b = each * _log(rng, 1, 8)
        while b * hkv * t * d > 1 << 28:
            t = t // 2 + 1
        return dict(base, B=b, T=t, each=each)
    b = _log(rng, 1, 32)
    while b * hkv * t * d > 1 << 28:
        b, t = (b + 1) // 2, t if b > 1 else t // 2 + 1
    return dict(base, B=b, T=t, kept=rng.randint(1, max(1, t // 4)))


# ---------------------------------------------------------------- sizes
def _rng(case, salt):
    return random.Random("%s %s %s %s" % (case["op"], case["T"], case["B"], salt))


def _counts(case, most, least=0, salt=0, seqs=None):
    """[B][Hkv] numbers of rows: `most` for the first sequence, fewer for some of the others (and their heads)."""
    rng, got = _rng(case, salt), []
    for b in range(seqs or case["B"]):
        n = most if b == 0 or case["ragged"] == "no" else max(least, most - rng.randint(0, most // 2 + 1))
        got.append([n if case["ragged"] != "heads" else max(least, n - rng.randint(0, n // 3))
                    for _ in range(case["Hkv"])])
    return got


def _starts(case):
    """Where the packed sequences begin, and the end of the last: any lengths, some of them 0 or 1."""
    rng = _rng(case, "starts")
    cuts = sorted(rng.randint(0, case["T"]) for _ in range(case["S"] - 1))
    return [0] + cuts + [case["T"]]


def _lengths(case):
    if not case["S"]:
        return [case["T"]] * case["B"]
    at = _starts(case)
    return [b - a for a, b in zip(at, at[1:])]


def _sizes(case):
    """(lens [B][Hkv], entries held [B], entries of a table row, pages of the pool) of a page case."""
    page, rng = case["page"], _rng(case, "pages")
    lens = _counts(case, case["T"], 1)
    held = [-(-max(row) // page) for row in lens]
    if case["op"] == "fork":                        # the sequences that are forked, and ended ones
        held = [n + rng.randint(0, 1) if b % case["each"] == 0 else rng.randint(0, 2) for b, n in enumerate(held)]
        lens = [row if b % case["each"] == 0 else [0] * case["Hkv"] for b, row in enumerate(lens)]
        new = 0
        for b in range(case["B"]):
            src = lens[b - b % case["each"]]
            new += -(-max(src) // page) - min(src) // page
        return lens, held, max(held) + 2, sum(held) + new + rng.randint(0, 5)
    if case["op"] == "compact":
        return lens, held, max(held) + 1, sum(held) + case["B"] * -(-case["kept"] // page) + rng.randint(0, 5)
    while sum(held) > case["n_pages"]:              # (hold: a pool that is nearly full)
        b = rng.randrange(case["B"])
        lens[b] = [n // 2 for n in lens[b]]
        held[b] = -(-max(lens[b]) // page)
    return lens, held, case["max_pages"], case["n_pages"]


def _wanted(case, lens):
    """[B][Hkv] rows to hold: a token more of most, none of ended ones, prompts of new ones."""
    rng, got = _rng(case, "want"), []
    for row in lens:
        x = rng.random()
        if x < 0.05:
            got.append([0] * len(row))
        elif x < 0.1:
            got.append([rng.randint(0, case["T"])] * len(row))
        else:
            got.append([n + 1 for n in row])
    return got


def _kept(case):
    return _counts(case, case["kept"], 0, "kept")


def _shared(case):
    """[G][Hkv] shared rows, [B][Hkv] rows with each sequence's own, [B] new tokens."""
    rng = _rng(case, "own")
    shared = _counts(case, case["T"], 0, "shared", case["G"])
    new = [case["n"] if b == 0 or case["ragged"] == "no" else rng.randint(min(1, case["n"]), case["n"])
           for b in range(case["B"])]
    mine = [case["own"] if case["ragged"] == "no" else rng.randint(case["n"], case["own"]) for _ in range(case["B"])]
    each = case["B"] // case["G"]
    return shared, [[x + mine[b] for x in shared[b // each]] for b in range(case["B"])], new


def _row_bytes(case):
    """Bytes of one cached row of K and V with their scales."""
    return 2 * (case["d"] * (2 if case["cache"] == "bf16" else 1) + (0 if case["cache"] == "bf16" else 4))


def work(case):
    b, d = case["B"], case["d"]
    if case["op"] == "prompt":
        pairs = sum(n * (n + 1) // 2 if case["causal"] else n * n for n in _lengths(case))
        rows = b * case["T"]
        return {"bytes": 4 * rows * d * (case["Hq"] + case["Hkv"]) + (4 * rows * case["Hq"] if case["lse"] else 0),
                "flops": 4 * d * case["Hq"] * pairs}
    if case["op"] == "shared":
        shared, lens, new = _shared(case)
        each, gh = b // case["G"], case["Hq"] // case["Hkv"]
        rows, seen = sum(map(sum, shared)), 0
        for i, row in enumerate(lens):
            rows += sum(x - y for x, y in zip(row, shared[i // each]))
            for length in row:
                seen += sum(max(0, length - new[i] + j + 1) if case["causal"] else length for j in range(new[i]))
        return {"bytes": rows * _row_bytes(case) + 4 * b * case["Hq"] * case["n"] * d, "flops": 4 * d * gh * seen}
    lens, held, most, pages = _sizes(case)
    book = 4 * (2 * b * most + pages)
    if case["op"] == "hold":
        return {"bytes": book + 4 * b * case["Hkv"], "flops": b * most}
    rows = 0
    if case["op"] == "compact":
        rows = sum(map(sum, _kept(case)))
        return {"bytes": book + rows * (4 + 2 * _row_bytes(case)), "flops": rows}
    for i in range(b):
        src = lens[i - i % case["each"]]
        if i % case["each"]:
            rows += sum(n - min(src) // case["page"] * case["page"] for n in src)
    return {"bytes": book + 2 * rows * _row_bytes(case), "flops": rows}


# ---------------------------------------------------------------- inputs
def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV)


def _int32(rows):
    return torch.tensor(rows, dtype=torch.int32, device=DEV)


def _tokens(x, layout):
    """[B, H, T, d] as given, or a view of a tensor whose tokens come first, as a projection leaves them."""
    return x.transpose(1, 2).contiguous().transpose(1, 2) if layout == "tokens" else x


def _keys(gen, n, heads, t, d):
    """Keys with a few channels of large values, and values with a mean of their own in each channel."""
    k = _randn(gen, n, heads, t, d)
    k += torch.where(torch.rand((1, heads, 1, d), generator=gen, device=DEV) < 0.05, 4.0, 0.0)
    return k, _randn(gen, n, heads, t, d).add_(_randn(gen, 1, heads, 1, d), alpha=0.5)


def _quantise(x, cache):
    """Rows x [..., d] fp32 as a cache holds them: (values, scales or None)."""
    if cache == "bf16":
        return x.to(torch.bfloat16), None
    a = x.abs().amax(-1, keepdim=True)
    if cache == "e4m3":                            # the smallest power of two that brings the row within 448
        f, e = torch.frexp(a)
        e = (e - 9 + (f > 0.875)).clamp(min=-126)
        return (x * torch.ldexp(torch.ones_like(a), -e)).to(torch.float8_e4m3fn), torch.ldexp(torch.ones_like(a), e)[..., 0]
    a = a.clamp(min=2.0 ** -100)
    most = torch.full_like(a, 127.0)
    return torch.round(x * (most / a)).to(torch.int8), (a / most)[..., 0]


def _raw(pages):
    return pages.view(torch.uint8) if pages.dtype == torch.float8_e4m3fn else pages


def _pool(s, gen, pages):
    case = s["case"]
    for name, x in zip(("k", "v"), _keys(gen, pages, case["Hkv"], case["page"], case["d"])):
        s[name], s[name + "_scale"] = _quantise(x, case["cache"])


def _book(s, gen, lens, held, most, pages):
    """The table, the entries that name each page and the lengths, side by side in one tensor: what a
    program copies to try something and take it back."""
    order = torch.randperm(pages, generator=gen, device=DEV).tolist()
    table, at = [], 0
    for b, n in enumerate(held):
        table.append(order[at:at + n] + [-1] * (most - n))
        at += n
    if s["case"]["op"] == "compact":               # every second sequence has its first pages from the one before
        for b in range(1, len(table), 2):
            n = min(min(lens[b]), min(lens[b - 1])) // s["case"]["page"] // 2
            table[b][:n] = table[b - 1][:n]
    refs = [0] * pages
    for row in table:
        for p in row:
            if p >= 0:
                refs[p] += 1
    parts = (torch.tensor(table), torch.tensor(refs), torch.tensor(lens))
    s["saved"] = torch.cat([x.flatten() for x in parts]).to(DEV, torch.int32)
    s["book"] = s["saved"].clone()
    at = 0
    for name, x in zip(("table", "refs", "lens"), parts):
        s[name] = s["book"][at:at + x.numel()].view(x.shape)
        at += x.numel()


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed((seed * 7919 + 53) & 0x7FFFFFFF)
    s = dict(case=case)
    if case["op"] == "prompt":
        k, v = _keys(gen, case["B"], case["Hkv"], case["T"], case["d"])
        q = 1.5 * _randn(gen, case["B"], case["Hq"], case["T"], case["d"])
        s["q"], s["k"], s["v"] = (_tokens(x.to(torch.bfloat16), case["layout"]) for x in (q, k, v))
        s["starts"] = _int32(_starts(case)) if case["S"] else None
        return s
    if case["op"] == "shared":
        shared, lens, new = _shared(case)
        page, each = case["page"], case["B"] // case["G"]
        most = -(-max(map(max, lens)) // page) + 1
        firsts = [-(-max(row) // page) for row in shared]
        rows, fresh, copies, table = sum(firsts), 0, [], []
        for b, row in enumerate(lens):             # shared pages, copies of those it goes on to fill, its own
            g = b // each
            whole, held, first = min(shared[g]) // page, -(-max(row) // page), sum(firsts[:g])
            mine = [rows + fresh + j for j in range(held - whole)]
            copies += [(first + j, mine[j - whole]) for j in range(whole, firsts[g])]
            fresh += len(mine)
            table.append([first + j for j in range(whole)] + mine + [0] * (most - held))
        order = torch.randperm(rows + fresh + 3, generator=gen, device=DEV)
        _pool(s, gen, rows + fresh + 3)
        s["table"] = order[torch.tensor(table, device=DEV)].to(torch.int32)
        s["shared_table"] = s["table"][::each].contiguous()
        if copies:                                 # (the prompt's own pages are those of the first answer)
            src, dst = (order[torch.tensor(x, device=DEV)] for x in zip(*copies))
            for name in ("k", "v", "k_scale", "v_scale"):
                if s[name] is not None:
                    _raw(s[name])[dst] = _raw(s[name])[src]
        s["shared"], s["lens"], s["new"] = _int32(shared), _int32(lens), _int32(new)
        q = 1.5 * _randn(gen, case["B"], case["Hq"], case["n"], case["d"])
        s["q"] = _tokens(q.to(torch.bfloat16), case["layout"])
        return s
    lens, held, most, pages = _sizes(case)
    _pool(s, gen, pages)
    _book(s, gen, lens, held, most, pages)
    if case["op"] == "hold":
        s["rows"] = _int32(_wanted(case, lens))
    elif case["op"] == "fork":
        s["src"] = _int32([b - b % case["each"] for b in range(case["B"])])
    else:                                          # ascending rows, -1 behind each head's number of them
        s["counts"] = torch.minimum(_int32(_kept(case)), s["lens"])
        t = torch.arange(case["T"], device=DEV)
        pick = torch.rand((case["B"], case["Hkv"], case["T"]), generator=gen, device=DEV)
        pick = pick.masked_fill_(t >= s["lens"][..., None], 2.0).argsort(-1)[..., :case["kept"]]
        last = torch.arange(pick.shape[-1], device=DEV) >= s["counts"][..., None]
        pick = pick.masked_fill(last, case["T"]).sort(-1).values
        s["idx"] = torch.where(last, -1, pick).to(torch.int32)
    return s


# ---------------------------------------------------------------- plain forms
def _prompt(s):
    case, t = s["case"], s["case"]["T"]
    gh, at = case["Hq"] // case["Hkv"], torch.arange(t, device=DEV)
    out = torch.empty_like(s["q"])
    lse = torch.empty((case["B"], case["Hq"], t), device=DEV)
    if s["starts"] is None:
        hidden = torch.zeros((t, t), dtype=torch.bool, device=DEV)
    else:                                          # the sequence of a token: the starts behind which it lies
        seq = (at[:, None] >= s["starts"].long()).sum(1)
        hidden = seq[:, None] != seq
    if case["causal"]:
        hidden |= at[:, None] < at
    for b in range(case["B"]):
        for c in range(case["Hkv"]):
            k, v = s["k"][b, c].float().t().contiguous(), s["v"][b, c].float()
            for h in range(c * gh, (c + 1) * gh):
                x = ((s["q"][b, h].float() * (1.0 / math.sqrt(case["d"]))) @ k).masked_fill_(hidden, -math.inf)
                most = x.amax(-1, keepdim=True)
                x = (x - most).exp_()
                total = x.sum(-1, keepdim=True)
                out[b, h] = ((x @ v) / total).to(torch.bfloat16)
                lse[b, h] = (most + total.log())[:, 0]
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def _named(s):
    return (s["table"] >= 0) & (s["table"] < s["refs"].numel())


def _new_pages(s, want):
    """Free pages, lowest first, for the wanted places [B, max_pages], as long as they last: (places, pages, missing)."""
    free = (s["refs"] == 0).nonzero()[:, 0]
    number = want.sum(1)
    upto = number.cumsum(0)
    ok = (upto <= free.numel()) | (number == 0)
    take = want & ok[:, None]
    rank = (upto - number)[:, None] + want.cumsum(1) - 1
    return take, free[rank[take]].to(torch.int32), torch.where(ok, 0, number).to(torch.int32)


def _count(s, pages, by):
    s["refs"].index_add_(0, pages.long(), torch.full_like(pages, by))


def _copy_rows(s, at, into):
    """Pool rows `into` become rows `at` (-1: zeros, scale 1)."""
    for name in ("k", "v"):
        rows = _raw(s[name]).view(-1, s["case"]["d"])
        rows[into] = rows[at.clamp(min=0)].masked_fill((at < 0)[:, None], 0)
        scale = s[name + "_scale"]
        if scale is not None:
            scale.view(-1)[into] = torch.where(at < 0, 1.0, scale.view(-1)[at.clamp(min=0)])


def _slots(s, table, rows):
    """Row numbers in a pool seen as [-1, d] of the cached rows `rows` [B, Hkv, n]."""
    case = s["case"]
    page = case["page"]
    at = torch.take_along_dim(table.long()[:, None], (rows // page).clamp(max=table.shape[1] - 1), 2)
    head = torch.arange(case["Hkv"], device=DEV)[None, :, None]
    return (at * case["Hkv"] + head) * page + rows % page


def _all(s, missing):
    got = {n: s[n] for n in ("table", "refs", "lens", "k", "v", "k_scale", "v_scale")}
    return dict(got, missing=missing)


def _hold(s):
    page, most = s["case"]["page"], s["table"].shape[1]
    need = ((s["rows"].amax(1).clamp(min=0) + page - 1) // page).clamp(max=most)[:, None]
    j, named = torch.arange(most, device=DEV), _named(s)
    take, pages, missing = _new_pages(s, (j < need) & ~named)
    _count(s, s["table"][named & (j >= need)], -1)
    s["table"].masked_fill_(j >= need, -1)
    s["table"][take] = pages
    _count(s, pages, 1)
    return {"table": s["table"], "refs": s["refs"], "missing": missing}


def _fork(s):
    case, page, most = s["case"], s["case"]["page"], s["table"].shape[1]
    b, j, named = torch.arange(case["B"], device=DEV), torch.arange(most, device=DEV), _named(s)
    src = s["src"].long()
    moves = (src >= 0) & (src < case["B"]) & (src != b)
    src = torch.where(moves, src, b)
    lens = s["lens"][src]
    whole = (lens.amin(1) // page)[:, None]
    used = (lens.amax(1) + page - 1)[:, None] // page
    theirs = torch.where(named, s["table"], -1)[src]
    take, pages, missing = _new_pages(s, moves[:, None] & (j >= whole) & (j < used) & (theirs >= 0))
    moves &= missing == 0
    table = torch.where((j < whole), theirs, -1)
    table[take] = pages
    at = _slots(s, theirs, torch.arange(most * page, device=DEV).expand(case["B"], case["Hkv"], -1))
    into = _slots(s, table, torch.arange(most * page, device=DEV).expand(case["B"], case["Hkv"], -1))
    here = take.repeat_interleave(page, 1)[:, None] & (torch.arange(most * page, device=DEV) < lens[..., None])
    _copy_rows(s, at[here], into[here])
    _count(s, s["table"][moves[:, None] & named], -1)
    _count(s, table[moves[:, None] & (table >= 0)], 1)
    s["table"].copy_(torch.where(moves[:, None], table, s["table"]))
    s["lens"].copy_(torch.where(moves[:, None], lens, s["lens"]))
    return _all(s, missing)


def _compact(s):
    case, page, most = s["case"], s["case"]["page"], s["table"].shape[1]
    j, named = torch.arange(most, device=DEV), _named(s)
    n = s["idx"].shape[-1]
    moves = s["counts"].amax(1) >= 0
    counts = s["counts"].clamp(0, n)
    need = ((counts.amax(1) + page - 1) // page)[:, None]
    take, pages, missing = _new_pages(s, moves[:, None] & (j < need))
    moves &= missing == 0
    table = torch.full_like(s["table"], -1)
    table[take] = pages
    idx = s["idx"].long()
    known = (idx >= 0) & (idx < s["lens"][..., None])
    at = torch.where(known, _slots(s, torch.where(named, s["table"], -1), idx.clamp(min=0)), -1)
    into = _slots(s, table, torch.arange(n, device=DEV).expand(case["B"], case["Hkv"], -1))
    here = moves[:, None, None] & (torch.arange(n, device=DEV) < counts[..., None])
    _copy_rows(s, at[here], into[here])
    _count(s, s["table"][moves[:, None] & named], -1)
    _count(s, pages, 1)
    s["table"].copy_(torch.where(moves[:, None], table, s["table"]))
    s["lens"].copy_(torch.where(moves[:, None], counts, s["lens"]))
    return _all(s, missing)


def _attend(s):
    case = s["case"]
    b, hkv, n, d = case["B"], case["Hkv"], case["n"], case["d"]
    gh, each, t = case["Hq"] // hkv, b // case["G"], case["T"] + case["own"]
    rows = torch.arange(t, device=DEV).expand(b, hkv, -1)
    shared = s["shared"].repeat_interleave(each, 0)[..., None]
    at = torch.where(rows < shared, _slots(s, s["shared_table"].repeat_interleave(each, 0), rows),
                     _slots(s, s["table"], rows))

    def cached(name):
        x = _raw(s[name]).view(-1, d)[at].view(s[name].dtype).float()
        scale = s[name + "_scale"]
        return x if scale is None else x * scale.view(-1)[at][..., None]

    i = torch.arange(n, device=DEV)[:, None]
    lens, new = s["lens"][..., None, None], s["new"][:, None, None, None]
    seen = (rows[..., None, :] < lens) & (i < new)
    if case["causal"]:
        seen = seen & (rows[..., None, :] <= lens - new + i)
    q = s["q"].float().reshape(b, hkv, gh * n, d) * (1.0 / math.sqrt(d))
    p = (q @ cached("k").transpose(2, 3).contiguous()).view(b, hkv, gh, n, t).masked_fill_(~seen[:, :, None], -math.inf)
    p -= p.amax(-1, keepdim=True).clamp(min=-3e38)
    p = p.exp_().view(b, hkv, gh * n, t)
    total = p.sum(-1, keepdim=True)
    o = (p @ cached("v")) / torch.where(total > 0, total, 1.0)
    return {"out": o.view(b, case["Hq"], n, d).to(torch.bfloat16)}


def _own(s):
    import paper_2607_22586_amd as mm

    case = s["case"]
    if case["op"] == "prompt":
        got = mm.prompt_attention(s["q"], s["k"], s["v"], starts=s["starts"], causal=case["causal"],
                                  with_lse=case["lse"])
        return {"out": got[0], "lse": got[1]} if case["lse"] else {"out": got}
    cache = mm.PagedCache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"], s.get("refs"))
    if case["op"] == "hold":
        return {"table": s["table"], "refs": s["refs"], "missing": mm.cache_hold(cache, s["rows"])}
    if case["op"] == "fork":
        return _all(s, mm.cache_fork(cache, s["src"], s["lens"]))
    if case["op"] == "compact":
        return _all(s, mm.cache_compact(cache, s["lens"], s["idx"], s["counts"]))
    out = mm.shared_attention(s["q"], cache, s["lens"], s["shared"], shared_table=s["shared_table"],
                              q_counts=s["new"], T=case["T"] + case["own"], shared_T=case["T"],
                              causal=case["causal"])
    return {"out": out}


def run(state):
    if "saved" in state:                           # the pages as they were before the last pass
        state["book"].copy_(state["saved"])
    if own:
        return _own(state)
    return {"prompt": _prompt, "hold": _hold, "fork": _fork, "compact": _compact, "shared": _attend}[
        state["case"]["op"]](state)


# ---------------------------------------------------------------- in 64 bits
def _exact_prompt(s):
    case = s["case"]
    gh = case["Hq"] // case["Hkv"]
    out = torch.zeros((case["B"], case["Hq"], case["T"], case["d"]), dtype=torch.float64, device=DEV)
    lse = torch.zeros(out.shape[:3], dtype=torch.float64, device=DEV)
    spans = list(zip(_starts(case), _starts(case)[1:])) if case["S"] else [(0, case["T"])]
    for b in range(case["B"]):
        for h in range(case["Hq"]):
            for lo, hi in spans:
                if lo == hi:
                    continue
                q, k, v = (x[lo:hi].double() for x in (s["q"][b, h], s["k"][b, h // gh], s["v"][b, h // gh]))
                x = q @ k.t().contiguous() / math.sqrt(case["d"])
                if case["causal"]:
                    x = torch.where(torch.ones_like(x, dtype=torch.bool).tril(), x, -math.inf)
                lse[b, h, lo:hi] = torch.logsumexp(x, -1)
                out[b, h, lo:hi] = torch.exp(x - lse[b, h, lo:hi, None]) @ v
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def _exact_pages(s):
    """Sequence by sequence and entry by entry, on lists."""
    case, page = s["case"], s["case"]["page"]
    table, refs, lens = (s[n].tolist() for n in ("table", "refs", "lens"))
    left = [p for p, n in enumerate(refs) if n == 0]
    old, old_lens, missing, copies = [list(r) for r in table], [list(r) for r in lens], [], []
    src = s["src"].tolist() if "src" in s else None
    idx, counts = (s[n].tolist() if n in s else None for n in ("idx", "counts"))
    wanted = s["rows"].tolist() if "rows" in s else None
    out_of = False

    def take(number):
        nonlocal out_of, left
        out_of = out_of or (number > len(left))
        if number and out_of:
            return None
        got, left = left[:number], left[number:]
        return got

    for b in range(case["B"]):
        new = list(old[b])
        if case["op"] == "hold":
            need = min(-(-max(wanted[b]) // page), len(new))
            gaps = [j for j in range(need) if new[j] < 0]
            got = take(len(gaps))
            for j, p in zip(gaps, got or ()):
                new[j] = p
            new[need:] = [-1] * (len(new) - need)
            missing.append(len(gaps) if got is None else 0)
        elif case["op"] == "fork":
            if src[b] == b:
                missing.append(0)
                continue
            theirs, n = old[src[b]], old_lens[src[b]]
            first, used = min(n) // page, -(-max(n) // page)
            got = take(used - first)
            missing.append(used - first if got is None else 0)
            if got is None:
                continue
            new = theirs[:first] + got + [-1] * (len(new) - used)
            for c in range(case["Hkv"]):
                copies += [(theirs[t // page], new[t // page], c, t % page, t % page)
                           for t in range(first * page, n[c])]
            lens[b] = list(n)
        else:
            n = counts[b]
            got = take(-(-max(n) // page))
            missing.append(-(-max(n) // page) if got is None else 0)
            if got is None:
                continue
            new = got + [-1] * (len(new) - len(got))
            for c in range(case["Hkv"]):
                copies += [(old[b][t // page], new[i // page], c, t % page, i % page)
                           for i, t in enumerate(idx[b][c][:n[c]])]
            lens[b] = list(n)
        for p in old[b]:
            refs[p] -= p >= 0
        for p in new:
            refs[p] += p >= 0
        table[b] = new
    got = dict(table=torch.tensor(table, device=DEV), refs=torch.tensor(refs, device=DEV),
               missing=torch.tensor(missing, device=DEV))
    if case["op"] == "hold":
        return got
    got["lens"] = torch.tensor(lens, device=DEV)
    p0, p1, c, t0, t1 = torch.tensor(copies, device=DEV).view(-1, 5).t()
    for name in ("k", "v"):
        x = _raw(s[name]).clone()
        x[p1, c, t1] = x[p0, c, t0]
        got[name] = x.view(s[name].dtype).double()
        x = s[name + "_scale"]
        got[name + "_scale"] = None if x is None else x.double()
        if x is not None:
            got[name + "_scale"][p1, c, t1] = got[name + "_scale"][p0, c, t0]
    return got


def _exact_shared(s):
    case, page = s["case"], s["case"]["page"]
    each, gh = case["B"] // case["G"], case["Hq"] // case["Hkv"]
    out = torch.zeros((case["B"], case["Hq"], case["n"], case["d"]), dtype=torch.float64, device=DEV)
    shared, lens, new = (s[n].tolist() for n in ("shared", "lens", "new"))
    for b in range(case["B"]):
        for c in range(case["Hkv"]):
            n, rows = lens[b][c], shared[b // each][c]
            kv = []
            for name in ("k", "v"):
                parts = []
                for table, lo, hi in ((s["shared_table"][b // each], 0, min(rows, n)), (s["table"][b], rows, n)):
                    t = torch.arange(lo, max(lo, hi), device=DEV)
                    at = table.long()[t // page]
                    x = _raw(s[name])[at, c, t % page].view(s[name].dtype).double()
                    if s[name + "_scale"] is not None:
                        x = x * s[name + "_scale"][at, c, t % page].double()[:, None]
                    parts.append(x)
                kv.append(torch.cat(parts))
            q = s["q"][b, c * gh:(c + 1) * gh, :new[b]].double()
            x = (q.reshape(-1, case["d"]) @ kv[0].t().contiguous() / math.sqrt(case["d"])).view(gh, new[b], n)
            if case["causal"]:
                last = n - new[b] + torch.arange(new[b], device=DEV)[:, None]
                x = x.masked_fill(torch.arange(n, device=DEV) > last, -math.inf)
            if n:
                p = torch.nan_to_num(torch.softmax(x, -1)).view(-1, n)
                out[b, c * gh:(c + 1) * gh, :new[b]] = (p @ kv[1]).view(gh, new[b], case["d"])
    return {"out": out}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "prompt":
        return _exact_prompt(s)
    if case["op"] == "shared":
        return _exact_shared(s)
    return _exact_pages(s)
