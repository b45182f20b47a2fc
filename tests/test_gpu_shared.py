"""Attention of a batch whose sequences share leading rows, against its plain 64-bit form."""
import random

import numpy as np
import pytest
import torch

import paper_2607_22586_amd as mm
from shared import attention

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = (torch.bfloat16, torch.float8_e4m3fn, torch.int8)


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def problem(B, G, Hq, Hkv, d, dtype, page, prefix, own, n, seed, layout="heads", poison=True):
    """(cache, q, lens, shared, shared_table): rows of shared pages and own ones, written as the cache holds them;
    what must not be read (own rows below the shared ones, rows behind the lengths) is NaN or names no page."""
    rng = random.Random(seed)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    each = B // G
    shared = [[rng.choice((prefix, rng.randint(0, prefix))) for _ in range(Hkv)] for _ in range(G)]
    shared[0][0] = prefix
    mine = [rng.choice((own, rng.randint(0, own))) for _ in range(B)]
    lens = [[shared[b // each][c] + mine[b] for c in range(Hkv)] for b in range(B)]
    T = prefix + own + 1
    most = -(-T // page) + 1
    n_pages = (B + G) * most
    cache = mm.PagedCache.pool(B, Hkv, n_pages, most, d, dtype, page)
    order = list(range(n_pages))
    rng.shuffle(order)
    everyone = torch.tensor(order, dtype=torch.int32, device=DEV).view(B + G, most)
    # all rows of all pages random first, then what nobody may see made NaN
    flat = mm.PagedCache(cache.k, cache.v, cache.k_scale, cache.v_scale, everyone)
    k, v = (torch.randn((B + G, Hkv, most * page, d), generator=g, device=DEV) for _ in range(2))
    k += torch.where(torch.rand((1, Hkv, 1, d), generator=g, device=DEV) < 0.05, 4.0, 0.0)
    if poison:
        at = torch.arange(most * page, device=DEV)
        low, high = int32([[0] * Hkv] * G + [shared[b // each] for b in range(B)]), int32(shared + lens)
        hide = (at < low[..., None]) | (at >= high[..., None])
        k = k.masked_fill(hide[..., None], float("nan"))
        v = v.masked_fill(hide[..., None], float("nan"))
    mm.cache_write(flat, k, v)
    shared_table, table = everyone[:G].contiguous(), everyone[G:].contiguous()
    if poison:                                     # entries of whole pages before and behind name none
        for b in range(B):
            first, last = min(shared[b // each]) // page, -(-max(lens[b]) // page)
            table[b, :first] = rng.choice((-1, n_pages, 1 << 30))
            table[b, last:] = -1
    cache.table.copy_(table)
    q = 1.5 * torch.randn((B, Hq, n, d), generator=g, device=DEV)
    q = q.bfloat16()
    if layout == "tokens":
        q = q.transpose(1, 2).contiguous().transpose(1, 2)
    return cache, q, int32(lens), int32(shared), shared_table


def check(got, cache, q, lens, shared, table, **kw):
    out, tol = attention(cache, q, lens, shared, table, **kw)
    got = got.cpu().double().numpy()
    assert np.isfinite(got).all()
    err = np.abs(got - out)
    assert (err <= tol).all(), (err / np.maximum(tol, 1e-30)).max()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("B,G,Hq,Hkv,d,page,prefix,own,n", [
    (1, 1, 1, 1, 64, 16, 1, 1, 1),                 # as small as it gets
    (2, 1, 7, 1, 128, 64, 130, 5, 1),              # few rows in both parts
    (6, 2, 4, 2, 64, 32, 100, 40, 2),
    (8, 2, 28, 4, 128, 64, 333, 70, 1),            # 28 shared rows
    (5, 5, 4, 4, 64, 16, 65, 64, 3),               # groups of one
    (15, 1, 16, 2, 64, 16, 203, 33, 4),            # many shared rows, few own
    (12, 3, 32, 8, 128, 128, 300, 130, 5),
    (3, 1, 30, 1, 128, 64, 150, 90, 4),            # many rows in both parts
    (4, 2, 130, 2, 64, 64, 70, 80, 1),
    (32, 1, 4, 4, 128, 256, 700, 300, 1),
    (12, 1, 8, 1, 64, 64, 500, 3000, 1),           # own rows that are split, after many shared ones
    (3, 1, 14, 2, 128, 64, 200, 2500, 1),          # ... and few
    (70, 1, 28, 4, 128, 64, 900, 100, 1),          # a launch for each part, the own one joins
    (40, 2, 40, 1, 64, 32, 600, 70, 2),            # ... with many own rows
    (300, 2, 2, 1, 64, 16, 100, 40, 1)])
def test_shared_attention(dtype, causal, B, G, Hq, Hkv, d, page, prefix, own, n):
    cache, q, lens, shared, table = problem(B, G, Hq, Hkv, d, dtype, page, prefix, own, n, B + n, "tokens")
    got = mm.shared_attention(q, cache, lens, shared, table, causal=causal)
    check(got, cache, q, lens, shared, table, causal=causal)
    # closer bounds, and one that is too small for the prefix by nothing
    got = mm.shared_attention(q, cache, lens, shared, table, causal=causal, T=int(lens.max()), shared_T=prefix)
    check(got, cache, q, lens, shared, table, causal=causal)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,d,n", [(4, 2, 64, 3), (32, 2, 128, 5), (8, 1, 128, 9)])
def test_drafted_tokens_of_some(dtype, Hq, Hkv, d, n):
    """Sequences with fewer queries than others, and with none."""
    B, G = 6, 2
    cache, q, lens, shared, table = problem(B, G, Hq, Hkv, d, dtype, 32, 90, 50, n, n)
    counts = [n, 0, 1, n + 5, -3, n - 1]
    for causal in (True, False):
        got = mm.shared_attention(q, cache, lens, shared, table, q_counts=int32(counts), causal=causal)
        check(got, cache, q, lens, shared, table, q_counts=counts, causal=causal)
        for b, m in enumerate(counts):
            assert bool((got[b, :, max(0, min(m, n)):] == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,n", [(4, 1), (4, 6), (80, 2)])
def test_sequences_of_fewer_rows_than_are_shared(dtype, Hq, n):
    """Lengths below the shared rows, of no rows at all, and chunks that reach back into the shared rows."""
    B, G, Hkv, d = 8, 2, 1, 64
    cache, q, lens, shared, table = problem(B, G, Hq, Hkv, d, dtype, 16, 100, 20, n, 5, poison=False)
    lens = int32([[100], [0], [37], [1], [103], [64], [99], [-5]])
    shared = int32([[100], [70]])
    for causal in (True, False):
        got = mm.shared_attention(q, cache, lens, shared, table, causal=causal)
        check(got, cache, q, lens, shared, table, causal=causal)
    none = mm.shared_attention(q, cache, lens * 0, shared, table)
    assert bool((none == 0).all())
    nothing = int32([[0], [-4]])                   # no shared rows: what chunk_attention gives
    got = mm.shared_attention(q, cache, lens, nothing, table)
    check(got, cache, q, lens, nothing, table)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,Hq,T", [(2, 2, 9000), (24, 8, 3000)])
def test_long_prefixes_key_by_key(dtype, B, Hq, T):
    """All but e^-32 of a query's weight on one key of the prefix in turn: none is left out or counted twice.

    Key t is its 14 bits as -1 and 1, the query 128 times them, so that a key j bits away has e^(-32 j) times the
    weight: together less than 14 e^-32 1.001 < 1.8e-13, of values at most 14 away: 2.6e-12.  Beside it the result
    is rounded to bf16, as `want` is (u each), and for int8 the weight times V's scale too (u)."""
    d, page = 64, 64
    cache = mm.PagedCache.empty(1, 1, T, d, dtype, page)
    bits = (torch.arange(T, device=DEV)[:, None] >> torch.arange(14, device=DEV)) & 1
    k = torch.zeros((1, 1, T, d), device=DEV)
    k[0, 0, :, :14] = (bits * 2 - 1).float()
    v = torch.randint(-7, 8, (1, 1, T, d), device=DEV).float()
    mm.cache_write(cache, k, v)
    want = mm.cache_read(cache, int32([[T]]), T, torch.float32)[1][0, 0].bfloat16()
    many = mm.PagedCache(cache.k, cache.v, cache.k_scale, cache.v_scale, torch.full((B, cache.table.shape[1]), -1,
                                                                                     dtype=torch.int32, device=DEV))
    lens, shared = int32([[T]] * B), int32([[T]])
    for lo in range(0, T, B * Hq * 4):
        at = (lo + torch.arange(B * Hq * 4, device=DEV)).clamp(max=T - 1)
        q = (8 * 16 * k[0, 0, at]).bfloat16().view(B, 4, Hq, d).transpose(1, 2).contiguous()
        got = mm.shared_attention(q, many, lens, shared, cache.table, causal=False)
        off = (got.transpose(1, 2).reshape(-1, d).double() - want[at].double()).abs()
        assert bool((off <= 3 * 2.0 ** -8 * want[at].double().abs() + 2.6e-12).all())


def test_as_chunk_attention_on_a_forked_cache():
    """A prompt in a pool, forked, a token appended to each answer: both calls see the same rows."""
    B, Hq, Hkv, d, page = 8, 14, 2, 128, 32
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    for dtype in TYPES:
        cache = mm.PagedCache.pool(B, Hkv, 150, 12, d, dtype, page)
        lens = torch.zeros((B, Hkv), dtype=torch.int32, device=DEV)
        lens[0], lens[4] = int32([300, 211]), int32([64, 96])
        mm.cache_hold(cache, lens)
        k, v = (torch.randn((B, Hkv, 300, d), generator=g, device=DEV).bfloat16() for _ in range(2))
        mm.cache_write(cache, k, v, counts=lens)
        shared = lens[::4].contiguous()
        assert int(mm.cache_fork(cache, int32([0] * 4 + [4] * 4), lens).sum()) == 0
        for step in range(3):
            assert int(mm.cache_hold(cache, lens + 1).sum()) == 0
            k, v = (torch.randn((B, Hkv, 1, d), generator=g, device=DEV).bfloat16() for _ in range(2))
            mm.cache_write(cache, k, v, start=lens)
            lens += 1
            q = torch.randn((B, Hq, 1, d), generator=g, device=DEV).bfloat16()
            got = mm.shared_attention(q, cache, lens, shared)
            check(got, cache, q, lens, shared, cache.table[::4].contiguous())
            other = mm.chunk_attention(q, cache, lens).float()
            assert float((got.float() - other).abs().max()) <= 2 ** -7 * float(other.abs().max())


def test_captured_on_another_stream_with_its_own_workspace():
    """Two graphs with workspaces of their own, replayed in turn as lengths grow."""
    args = [problem(6, 2, 14, 2, 128, torch.float8_e4m3fn, 64, 200, 60, 1, s) for s in (1, 2)]
    stream, graphs = torch.cuda.Stream(), []
    for cache, q, lens, shared, table in args:
        ws = torch.empty(mm.shared_attention_workspace(6, 14, 2, 261, 128, 1, 2), dtype=torch.uint8, device=DEV)
        out, graph = torch.empty_like(q), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            mm.shared_attention(q, cache, lens, shared, table, T=261, shared_T=200, workspace=ws, out=out)
        graphs.append((graph, out, ws))
    for turn in range(3):
        for graph, out, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for (cache, q, lens, shared, table), (_, out, _) in zip(args, graphs):
            check(out, cache, q, lens, shared, table)
            lens -= (lens > shared.repeat_interleave(3, 0)).int()
            q.copy_(torch.randn(q.shape, device=DEV).bfloat16())


def test_strides_of_q_and_out():
    cache, q, lens, shared, table = problem(4, 1, 6, 2, 64, torch.bfloat16, 16, 70, 20, 3, 8)
    want = mm.shared_attention(q, cache, lens, shared, table)
    big = torch.full((4, 3, 8, 80), 5.0, dtype=torch.bfloat16, device=DEV)
    big[:, :, 1:7, 8:72] = q.transpose(1, 2)
    view = big[:, :, 1:7, 8:72].transpose(1, 2)
    out = torch.full((4, 7, 5, 72), 3.0, dtype=torch.bfloat16, device=DEV)
    got = mm.shared_attention(view, cache, lens, shared, table, out=out[:, :6, 1:4, 8:])
    assert torch.equal(got, want)
    out[:, :6, 1:4, 8:] = 3.0
    assert bool((out == 3.0).all())
