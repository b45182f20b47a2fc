"""Forks and compactions of tables, pools, heads and batches that one workgroup does not plan, against their plain
form: every bit of the pools, the table, the counters and the lengths."""
import random

import pytest
import torch

import paper_2607_22586_amd as mm
from book import Book, copy_of
from test_gpu_pages import assign, check, count, filled, int32

pytestmark = pytest.mark.gpu

# (B, Hkv, n_pages, max_pages, rows): just beyond each of the limits
SIZES = [(70, 1, 1200, 64, 100), (5, 2, 8203, 60, 150), (4, 65, 90, 8, 70), (1025, 1, 6000, 3, 40), (33, 3, 10001, 160, 90)]


def some_rows(rng, B, Hkv, T):
    out = []
    for _ in range(B):
        n = rng.choice((0, 1, 16, 17, T, rng.randint(0, T)))
        out.append([rng.choice((n, rng.randint(0, n))) for _ in range(Hkv)])
    return out


@pytest.mark.parametrize("B,Hkv,n_pages,most,T", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
def test_fork(dtype, B, Hkv, n_pages, most, T):
    rng = random.Random("large fork %s %s" % (B, most))
    cache = filled(B, Hkv, n_pages, most, 64, dtype, 16, rng)
    for turn in range(3):
        lens = some_rows(rng, B, Hkv, T)
        assign(cache, lens, rng, shared=turn == 1)
        if turn == 2:                              # a row that names no page, lengths past the table's row
            cache.table[0, 0] = n_pages
            count(cache)
            lens[B - 1][0] = most * 16 + 5
        rows = int32(lens)
        src = int32([(b + 1) % B if turn == 0 else rng.choice((b, rng.randrange(B), -1, B)) for b in range(B)])
        state = copy_of(cache, rows)
        want = Book(state).fork(src.cpu())
        check(cache, rows, state, mm.cache_fork(cache, src, rows), want)
        kept = cache.refs.clone()
        count(cache)
        assert torch.equal(kept, cache.refs)


@pytest.mark.parametrize("B,Hkv,n_pages,most,T", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
def test_compact(dtype, B, Hkv, n_pages, most, T):
    rng = random.Random("large compact %s %s" % (B, most))
    cache, n = filled(B, Hkv, n_pages, most, 64, dtype, 16, rng), 37
    for turn in range(3):
        lens = some_rows(rng, B, Hkv, T)
        assign(cache, lens, rng, shared=turn == 1)
        rows = int32(lens)
        idx = int32([[[rng.choice((rng.randint(0, T), rng.randint(0, T), -1, m, 1 << 30)) for _ in range(n)]
                      for m in row] for row in lens])
        counts = int32([[rng.choice((0, n, n + 9, rng.randint(0, n))) for _ in range(Hkv)] for _ in range(B)])
        counts[B // 2] = -1                        # stays as it is
        if turn == 2:
            counts = rows                          # the lengths themselves
        state = copy_of(cache, rows)
        want = Book(state).compact(idx.cpu(), counts.cpu())
        check(cache, rows, state, mm.cache_compact(cache, rows, idx, counts), want)
        kept = cache.refs.clone()
        count(cache)
        assert torch.equal(kept, cache.refs)


@pytest.mark.parametrize("B,Hkv,n_pages,most,T", SIZES)
def test_pools_that_run_out_between_two_sequences(B, Hkv, n_pages, most, T):
    """As many free pages as the first half of the sequences wants, and one more."""
    rng = random.Random("large few %s %s" % (B, most))
    cache = filled(B, Hkv, n_pages, most, 64, torch.bfloat16, 16, rng)
    for op in ("fork", "compact"):
        lens = [[x + 1 for x in row] for row in some_rows(rng, B, Hkv, T - 1)]
        assign(cache, lens, rng)
        rows, src = int32(lens), int32([(b + 1) % B for b in range(B)])
        idx = int32(list(range(20))).expand(B, Hkv, -1).contiguous()
        counts = int32([[rng.randint(1, 20) for _ in range(Hkv)] for _ in range(B)])

        def calls(book):
            return book.fork(src.cpu()) if op == "fork" else book.compact(idx.cpu(), counts.cpu())

        trial = copy_of(cache, rows)
        trial["table"], trial["refs"] = trial["table"].clone(), trial["refs"].clone()
        book, used = Book(trial), []
        take = book.take
        book.take = lambda m: used.append(m) or take(m)
        calls(book)
        free = (cache.refs == 0).nonzero()[:, 0]
        cache.refs[free[sum(used[:len(used) // 2]) + 1:]] = 1      # (held elsewhere)
        state = copy_of(cache, rows)
        want = calls(Book(state))
        assert any(want) and not all(want)
        got = mm.cache_fork(cache, src, rows) if op == "fork" else mm.cache_compact(cache, rows, idx, counts)
        check(cache, rows, state, got, want)

