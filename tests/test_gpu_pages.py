"""The calls that change a cache's pages against their plain form: every bit of the pools, the table, the counters
and the lengths."""
import random

import numpy as np
import pytest
import torch

import paper_2607_22586_amd as mm
from book import Book, copy_of
from paged import attention

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = (torch.bfloat16, torch.float8_e4m3fn, torch.int8)


def filled(B, Hkv, n_pages, most, d, dtype, page, rng):
    """A pool whose rows hold random bits (bf16 and e4m3 patterns of NaN among them: copies keep them)."""
    cache = mm.PagedCache.pool(B, Hkv, n_pages, most, d, dtype, page)
    g = torch.Generator(device=DEV)
    g.manual_seed(rng.randint(0, 1 << 30))
    for n in ("k", "v"):
        x = getattr(cache, n).view(torch.uint8)
        x.copy_(torch.randint(0, 256, x.shape, generator=g, device=DEV, dtype=torch.uint8))
        if dtype != torch.bfloat16:
            getattr(cache, n + "_scale").copy_(torch.rand(cache.k.shape[:3], generator=g, device=DEV) + 0.5)
    return cache


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def assign(cache, lens, rng, shared=False, extra=1):
    """Pages in random order for the rows of each sequence and up to `extra` more; every second sequence's
    first pages those of the one before, if asked for."""
    B, most = cache.table.shape
    page = cache.k.shape[2]
    order = list(range(cache.k.shape[0]))
    rng.shuffle(order)
    table, at = [], 0
    for b in range(B):
        n = min(most, -(-max(max(lens[b]), 0) // page) + rng.randint(0, extra))
        table.append(order[at:at + n] + [-1] * (most - n))
        assert len(table[b]) == most
        at += n
        if shared and b % 2:
            m = max(0, min(min(lens[b]), min(lens[b - 1]))) // page
            table[b][:m] = table[b - 1][:m]
    cache.table.copy_(torch.tensor(table, dtype=torch.int32))
    count(cache)


def count(cache):
    t = cache.table.cpu().numpy().ravel()
    n = cache.k.shape[0]
    cache.refs.copy_(torch.from_numpy(np.bincount(t[(t >= 0) & (t < n)], minlength=n).astype(np.int32)))


def check(cache, lens, state, got, want):
    assert got.tolist() == want
    after = copy_of(cache, lens)
    for n, x in state.items():
        if x is not None:
            y = after[n]
            if x.dtype == torch.bfloat16:
                x, y = x.view(torch.int16), y.view(torch.int16)
            assert torch.equal(x, y), n


@pytest.mark.parametrize("B,Hkv,n_pages,most,page,T", [
    (1, 1, 1, 1, 16, 16), (1, 1, 3, 5, 64, 200), (5, 2, 40, 9, 16, 130), (32, 4, 300, 24, 64, 700),
    (300, 1, 2500, 300, 16, 300), (7, 3, 5000, 700, 16, 9000)])
@pytest.mark.parametrize("seed", [0, 1])
def test_hold(B, Hkv, n_pages, most, page, T, seed):
    rng = random.Random("hold %s" % seed)
    cache = filled(B, Hkv, n_pages, most, 64, torch.bfloat16, page, rng)
    lens, left = [], n_pages
    for b in range(B):
        n = rng.randint(0, min(T, most * page, max(0, left - 1) * page))
        lens.append([rng.randint(0, n) for _ in range(Hkv)])
        left -= -(-max(lens[b]) // page) + 1
    assign(cache, lens, rng, extra=1 if left >= 0 else 0)
    if seed:                                       # entries that name no page within the rows
        cache.table[:, most // 2] = int32([rng.choice((-1, -7, n_pages, 1 << 30)) for _ in range(B)])
        count(cache)
    for _ in range(3):
        rows = int32([[rng.choice((n, n + 1, 0, -5, rng.randint(0, T), 1 << 30)) for n in row] for row in lens])
        state = copy_of(cache, None)
        want = Book(state).hold(rows.cpu())
        check(cache, None, state, mm.cache_hold(cache, rows), want)
        t = cache.table.cpu()
        count_of = np.bincount(t[t >= 0].numpy(), minlength=n_pages)
        assert (count_of == cache.refs.cpu().numpy()).all()


def test_hold_to_the_last_page_and_beyond():
    """A pool that just suffices, one that lacks a page, and sequences behind the one that lacks it."""
    cache = mm.PagedCache.pool(4, 1, 9, 4, 64, page=16)
    assert mm.cache_hold(cache, int32([[33], [64], [1], [16]])).tolist() == [0, 0, 0, 0]
    assert cache.table.tolist() == [[0, 1, 2, -1], [3, 4, 5, 6], [7, -1, -1, -1], [8, -1, -1, -1]]
    assert mm.cache_hold(cache, int32([[33], [0], [33], [16]])).tolist() == [0, 0, 2, 0]     # (freed by this call)
    assert cache.table.tolist() == [[0, 1, 2, -1], [-1] * 4, [7, -1, -1, -1], [8, -1, -1, -1]]
    assert mm.cache_hold(cache, int32([[64], [64], [16], [17]])).tolist() == [0, 4, 0, 1]
    assert cache.table.tolist() == [[0, 1, 2, 3], [-1] * 4, [7, -1, -1, -1], [8, -1, -1, -1]]
    assert cache.refs.tolist() == [1, 1, 1, 1, 0, 0, 0, 1, 1]


def test_hold_in_a_pool_of_more_pages_than_one_round_of_chunks():
    n = 600_011
    cache = mm.PagedCache.pool(3, 1, n, 5000, 64, torch.int8, 16)
    cache.refs.fill_(1)
    free = sorted(random.Random(5).sample(range(n), 4000) + [n - 1])
    cache.refs[torch.tensor(free, device=DEV)] = 0
    free = [p for p in range(n) if p in set(free)]
    got = mm.cache_hold(cache, int32([[16 * 1000], [16 * 2000], [16 * (len(free) - 3000)]]))
    assert got.tolist() == [0, 0, 0]
    t = cache.table.tolist()
    assert t[0][:1000] + t[1][:2000] + t[2][:len(free) - 3000] == free
    assert (cache.refs == 1).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,Hkv,d,page,T", [(2, 1, 64, 16, 40), (6, 2, 64, 32, 150), (5, 3, 128, 16, 100),
                                            (9, 2, 128, 64, 200)])
@pytest.mark.parametrize("ragged", [False, True])
def test_fork(dtype, B, Hkv, d, page, T, ragged):
    rng = random.Random("fork %s %s %s" % (B, page, ragged))
    most = -(-T // page) + 1
    cache = filled(B, Hkv, 4 * B * most, most, d, dtype, page, rng)
    for turn in range(4):
        lens = []
        for b in range(B):
            n = rng.choice((0, 1, page, page + 1, T, rng.randint(0, T), most * page))
            lens.append([rng.randint(0, n) if ragged else n for _ in range(Hkv)])
        assign(cache, lens, rng, shared=turn % 2 == 1)
        if turn == 3:                              # a source with an entry that names no page, one with lengths past its row
            cache.table[0, 0] = -1
            count(cache)
            lens[B - 1][0] = most * page + 5
        rows = int32(lens)
        src = int32([rng.choice((b, rng.randrange(B), rng.randrange(B), -1, B)) for b in range(B)])
        if turn == 0:                              # sources that are replaced themselves
            src = int32([(b + 1) % B for b in range(B)])
        state = copy_of(cache, rows)
        want = Book(state).fork(src.cpu())
        check(cache, rows, state, mm.cache_fork(cache, src, rows), want)
        count_before = cache.refs.clone()
        count(cache)
        assert torch.equal(count_before, cache.refs)


@pytest.mark.parametrize("short", [0, 1, 3])
def test_fork_with_few_free_pages(short):
    rng = random.Random(3)
    B, page, most = 6, 16, 4
    cache = filled(B, 2, B * most, most, 64, torch.float8_e4m3fn, page, rng)
    lens = [[33, 20], [0, 0], [0, 0], [16, 16], [5, 48], [0, 0]]
    assign(cache, lens, rng, extra=0)
    free = (cache.refs == 0).nonzero()[:, 0]
    cache.refs[free[5 - short:]] = 1               # (held elsewhere)
    held = cache.refs.clone()
    rows = int32(lens)
    src = int32([0, 0, 3, 3, 4, 4])                # 2, 0 and 3 pages
    state = copy_of(cache, rows)
    want = Book(state).fork(src.cpu())
    assert want == ([0] * 6 if short == 0 else [0, 0, 0, 0, 0, 3])
    check(cache, rows, state, mm.cache_fork(cache, src, rows), want)
    assert int(cache.refs.sum()) >= int(held.sum())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,Hkv,d,page,T,n", [(1, 1, 64, 16, 40, 1), (3, 2, 128, 16, 100, 37), (4, 3, 64, 64, 300, 130),
                                              (2, 1, 128, 128, 500, 257)])
def test_compact(dtype, B, Hkv, d, page, T, n):
    rng = random.Random("compact %s %s" % (B, page))
    most = -(-T // page) + 1
    cache = filled(B, Hkv, 4 * B * most, most, d, dtype, page, rng)
    for turn in range(4):
        lens = [[rng.choice((0, T, rng.randint(0, T))) for _ in range(Hkv)] for _ in range(B)]
        assign(cache, lens, rng, shared=turn % 2 == 1)
        if turn == 3:
            cache.table[0, 1] = 1 << 20
            count(cache)
        rows = int32(lens)
        counts = int32([[rng.choice((0, n, n + 9, rng.randint(0, n))) for _ in range(Hkv)] for _ in range(B)])
        if turn == 2:
            counts[B - 1] = -1                     # stays as it is
        # any rows: ascending ones, some twice, some that are not there
        idx = int32([[sorted(rng.randint(0, max(0, m - 1)) for _ in range(n)) if turn == 0 else
                      [rng.choice((rng.randint(0, T), rng.randint(0, T), -1, m, 1 << 30)) for _ in range(n)]
                      for m in row] for row in lens])
        state = copy_of(cache, rows)
        want = Book(state).compact(idx.cpu(), counts.cpu())
        check(cache, rows, state, mm.cache_compact(cache, rows, idx, counts), want)
        kept = cache.refs.clone()
        count(cache)
        assert torch.equal(kept, cache.refs)


def test_compact_counts_are_the_lengths():
    """The lengths themselves as counts: every row in a new order."""
    rng = random.Random(1)
    cache = filled(3, 2, 40, 6, 64, torch.int8, 16, rng)
    lens = [[70, 33], [0, 5], [96, 96]]
    assign(cache, lens, rng, extra=0)
    rows = int32(lens)
    idx = torch.arange(95, -1, -1, dtype=torch.int32, device=DEV).expand(3, 2, -1).contiguous()
    state = copy_of(cache, rows)
    want = Book(state).compact(idx.cpu(), rows.cpu())
    check(cache, rows, state, mm.cache_compact(cache, rows, idx, rows), want)


def test_compact_more_rows_than_the_table_names():
    rng = random.Random(2)
    cache = filled(1, 1, 8, 2, 64, torch.bfloat16, 16, rng)
    assign(cache, [[32]], rng, extra=0)
    rows, counts = int32([[32]]), int32([[40]])
    idx = torch.arange(40, dtype=torch.int32, device=DEV).view(1, 1, 40)
    state = copy_of(cache, rows)
    want = Book(state).compact(idx.cpu(), counts.cpu())
    check(cache, rows, state, mm.cache_compact(cache, rows, idx, counts), want)


def test_compact_without_pages_keeps_all():
    rng = random.Random(4)
    cache = filled(2, 1, 7, 4, 64, torch.bfloat16, 16, rng)
    assign(cache, [[48], [48]], rng, extra=0)      # one page is free
    rows, counts = int32([[48], [48]]), int32([[17], [3]])
    idx = torch.arange(17, dtype=torch.int32, device=DEV).expand(2, 1, 17).contiguous()
    state = copy_of(cache, rows)
    want = Book(state).compact(idx.cpu(), counts.cpu())
    assert want == [2, 1]
    check(cache, rows, state, mm.cache_compact(cache, rows, idx, counts), want)


def tokens(B, Hkv, n, d, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return [torch.randn((B, Hkv, n, d), generator=g, device=DEV).bfloat16() for _ in range(2)]


@pytest.mark.parametrize("dtype", TYPES)
def test_a_prompt_answered_several_times(dtype):
    """Rows held, written, forked, grown apart, compacted and given back: every sequence attends to its own rows."""
    B, Hkv, d, page, T = 4, 2, 64, 16, 75
    cache = mm.PagedCache.pool(B, Hkv, 40, 8, d, dtype, page)
    lens = int32([[75, 40]] + [[0, 0]] * 3)
    assert mm.cache_hold(cache, lens).tolist() == [0] * 4
    k, v = tokens(B, Hkv, T, d, 1)
    mm.cache_write(cache, k, v, counts=lens)
    assert mm.cache_fork(cache, int32([0, 0, 0, 0]), lens).tolist() == [0] * 4
    assert lens.tolist() == [[75, 40]] * 4
    assert int((cache.table[:, :2] == cache.table[0, :2]).all()) and int((cache.refs == 4).sum()) == 2
    for step in range(8):
        assert mm.cache_hold(cache, lens + 1).tolist() == [0] * 4
        kn, vn = tokens(B, Hkv, 1, d, 10 + step)
        mm.cache_write(cache, kn, vn, start=lens)
        lens += 1
        k, v = (torch.cat([x, y], 2) for x, y in ((k, kn), (v, vn)))
    # what each sequence holds is what a cache of its own would
    own = mm.PagedCache.empty(B, Hkv, 100, d, dtype, page)
    rows = torch.arange(83, device=DEV)
    pick = torch.stack([torch.where(rows < n, rows, rows - n + 75) for n in (75, 40)])[None, :, :, None].expand(B, -1, -1, d)
    pick = pick.clamp(max=82)
    first = [x[:1].expand(B, -1, -1, -1).clone() for x in (k, v)]
    for x, y in zip(first, (k, v)):
        x[:, :, 75:] = y[:, :, 75:]
    mm.cache_write(own, *[torch.take_along_dim(x, pick, 2) for x in first], counts=lens)
    for x, y in zip(mm.cache_read(cache, lens, 100), mm.cache_read(own, lens, 100)):
        assert torch.equal(x, y)
    q = torch.randn((B, 4, 1, d), device=DEV).bfloat16()
    out, tol = attention(cache, q, lens)
    assert (abs(mm.chunk_attention(q, cache, lens, T=100).cpu().double().numpy() - out) <= tol).all()
    # compacted: the last 20 rows of sequences 1 and 3
    counts = int32([[-1, -1], [20, 20], [-1, -1], [20, 7]])
    before = mm.cache_read(cache, lens, 100)
    idx = (lens[..., None] - 20 + torch.arange(20, device=DEV)).to(torch.int32).contiguous()
    was = lens.clone()
    assert mm.cache_compact(cache, lens, idx, counts).tolist() == [0] * 4
    assert lens.tolist() == [was[0].tolist(), [20, 20], was[2].tolist(), [20, 7]]
    for x, y in zip(mm.cache_read(cache, lens, 100), before):
        assert torch.equal(x[0], y[0]) and torch.equal(x[2], y[2])
        for b, c, n in ((1, 0, 20), (1, 1, 20), (3, 0, 20), (3, 1, 7)):
            at = int(was[b, c]) - 20
            assert torch.equal(x[b, c, :n], y[b, c, at:at + n])
    mm.cache_hold(cache, torch.zeros_like(lens))
    assert int(cache.refs.abs().sum()) == 0 and int((cache.table != -1).sum()) == 0


def test_captured_and_replayed_on_another_stream():
    """hold, fork and compact in one graph: every replay goes on from the state that the one before left."""
    rng = random.Random(9)
    B, Hkv, page, most = 6, 2, 16, 6
    cache = filled(B, Hkv, 80, most, 64, torch.float8_e4m3fn, page, rng)
    lens = [[rng.randint(1, 60) for _ in range(Hkv)] for _ in range(B)]
    assign(cache, lens, rng)
    rows, src = int32(lens), int32([0, 0, 2, 2, 1, 5])
    counts = int32([[-1] * Hkv] * 3 + [[30, 9]] * 3)
    idx = torch.arange(31, -1, -1, dtype=torch.int32, device=DEV).expand(B, Hkv, -1).contiguous()
    ws = torch.empty(mm.cache_book_workspace(B, Hkv, 80, most), dtype=torch.uint8, device=DEV)
    out = [torch.empty(B, dtype=torch.int32, device=DEV) for _ in range(3)]

    def calls():
        mm.cache_hold(cache, rows, out[0], ws)
        mm.cache_fork(cache, src, rows, out[1], ws)
        mm.cache_compact(cache, rows, idx, counts, out[2], ws)

    state = copy_of(cache, rows)
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        calls()
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = [Book(state).hold(state["lens"]), Book(state).fork(src.cpu()), Book(state).compact(idx.cpu(), counts.cpu())]
        for x, y in zip(out, want):
            check(cache, rows, state, x, y)
        float(torch.randn(1000, device=DEV).sum())             # (the program's own work between replays)
