"""Attention over a paged cache, key by key: every key of a long cache carries half of some query's weight, so
that one that is missing, doubled or seen where it is not to be changes a result by as much as its size."""
import math

import numpy as np
import pytest
import torch

import paged
from paper_2607_22586_amd import binding as bd
from test_gpu_cache import BF16, DEV, KINDS, _gpu, check_attention, i32, make_cache, rnd  # noqa: F401

pytestmark = pytest.mark.gpu


def signs(seed, *shape):
    return (torch.randint(0, 2, shape, generator=torch.Generator().manual_seed(seed)) * 2 - 1).float()


def planted(B, Hkv, T, d, kind, page):
    """Keys and values of random signs.  At d = 128 a query of 3/2 of the sum of two keys has logits of about 17
    for them and, at more than four standard deviations, 9 for another: half of the weight each."""
    k, v = (signs(s, B, Hkv, T, d) for s in (1, 2))
    cache = make_cache(B, Hkv, T, d, kind, page)
    bd.cache_write(cache, k.to(DEV), v.to(DEV))
    return cache, k


def weights_matter(got, cache, q, lens, causal):
    """The result within its bound, far below the change of a result by a key of half the weight that is doubled
    (a third, in the dims where the two values differ), left out or seen against the mask (half or more)."""
    want, tol = paged.attention(cache, q, lens, None, causal)
    assert tol.max() < 0.1
    off = np.abs(got.cpu().double().numpy() - want)
    assert (off <= tol).all(), (off - tol).max()


# rows of a head: on the few-row kernel (of 1, 2 and 4 tiles of 16 rows) and the staged one (d = 64: fewer bytes a row)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,page,Gh,n", [(5001, 64, 1, 16), (4100, 16, 2, 16), (4999, 128, 4, 16), (5001, 64, 2, 64),
                                         (4100, 16, 1, 300)])
def test_every_key(kind, T, page, Gh, n):
    """Each key once with the one half a cache away, without a causal limit; keys of many splits."""
    Hkv, d = 4, 128
    cache, k = planted(1, Hkv, T, d, kind, page)
    lens = torch.full((1, Hkv), T, dtype=torch.int32)
    per = Hkv * Gh * n                             # keys of a call
    for first in range(0, T, per):
        at = (first + torch.arange(per)).view(Hkv, Gh * n) % T
        head = torch.arange(Hkv)[:, None]
        q = 1.5 * (k[0, head, at] + k[0, head, (at + T // 2) % T])
        q = q.view(1, Hkv * Gh, n, d).to(BF16)
        got = bd.chunk_attention(q.to(DEV), cache, lens.to(DEV), T=T, causal=False)
        weights_matter(got, cache, q, lens, False)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,page,Gh,n", [(4100, 16, 1, 16), (1000, 64, 1, 64), (2050, 64, 2, 150), (333, 32, 1, 333)])
def test_the_last_key_that_a_query_sees(kind, T, page, Gh, n):
    """Causal: a query aims at the last key that it sees and at the first that it does not."""
    Hkv, d = 2, 128
    cache, k = planted(1, Hkv, T, d, kind, page)
    lens = [[T, T - 37]]
    q = torch.empty(1, Hkv * Gh, n, d)
    for h in range(Hkv * Gh):
        c = h // Gh
        last = lens[0][c] - n + torch.arange(n)
        q[0, h] = 1.5 * (k[0, c, last.clamp(min=0)] + k[0, c, last + 1 - (last + 1 == T).int()])
    q = q.to(BF16)
    got = bd.chunk_attention(q.to(DEV), cache, i32(lens), T=T)
    weights_matter(got, cache, q, torch.tensor(lens, dtype=torch.int32), True)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("where", [0, 170, 250, 332])
def test_large_logits_in_staged_tiles(kind, d, where):
    """More than 64 rows of a head and a key of logits of several hundred: first, last, in each half of a tile."""
    T = 333
    cache = make_cache(1, 2, T, d, kind, 64)
    k, v = rnd(1, 1, 2, T, d) - 5.0, rnd(2, 1, 2, T, d)
    k[:, :, where] = 30.0
    bd.cache_write(cache, k.to(DEV), v.to(DEV))
    q = 3.0 + rnd(3, 1, 4, 40, d)
    for x in (q, -q):
        for causal in (True, False):
            check_attention(cache, x.to(BF16), [[T, T]], causal=causal)


@pytest.mark.parametrize("kind", KINDS)
def test_staged_tiles_past_32_bits(kind):
    """Pages behind 4 GiB of a pool (and, for bf16, 2^31 elements) under more than 64 rows of a head."""
    d, page, T = 128, 1024, 1500
    per_page = page * d * (2 if kind == BF16 else 1)
    n = (1 << 32) // per_page + 4
    raw_k, raw_v = (torch.empty((n, 1, page, d), dtype=torch.int16 if kind == BF16 else torch.uint8, device=DEV)
                    for _ in range(2))
    ks, vs = (None, None) if kind == BF16 else (torch.empty((n, 1, page), device=DEV) for _ in range(2))
    cache = bd.PagedCache(raw_k.view(kind), raw_v.view(kind), ks, vs, i32([[n - 1, n - 3]]))
    small = make_cache(1, 1, T, d, kind, 64)
    k, v = (rnd(s, 1, 1, T, d).to(DEV) for s in (8, 9))
    for x in (cache, small):
        bd.cache_write(x, k, v)
    q = rnd(4, 1, 5, 30, d, dtype=BF16).to(DEV)
    got = bd.chunk_attention(q, cache, i32([[T]]), T=T)
    assert torch.equal(got, bd.chunk_attention(q, small, i32([[T]]), T=T))
    check_attention(small, q, [[T]])
