"""Values at the ends of their range in the attention over a paged cache: infinities and NaN, sums near the
largest number, scales of every kind, against plain 64-bit forms (tests/paged.py)."""
import math

import numpy as np
import pytest
import torch

import paged
from paper_2607_22586_amd import binding as bd
from test_gpu_cache import BF16, DEV, E4M3, F32, I8, KINDS, _gpu, check_attention, i32, make_cache, rnd  # noqa: F401

pytestmark = pytest.mark.gpu

# (Hq, Hkv, T, n): rows of a head on the few-row kernel and on the staged one, over keys of one split and of
# many (they are more than the rows of a workgroup can walk before a join pays)
SPLITS = [(4, 2, 200, 2), (4, 2, 5000, 2), (8, 2, 200, 40), (8, 2, 5000, 40)]


def attend(cache, q, lens, q_counts=None, causal=True, T=None):
    print("attend", tuple(q.shape), cache.k.dtype, tuple(cache.k.shape), flush=True)
    return bd.chunk_attention(q.to(DEV), cache, i32(lens), None if q_counts is None else i32(q_counts), T=T,
                              causal=causal).cpu().float()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("Hq,Hkv,T,n", SPLITS)
def test_rows_that_are_not_there_beside_infinite_values(Hq, Hkv, T, n, causal):
    """Zeros for queries behind a sequence's count, whatever the rows of V that others see hold."""
    cache = make_cache(2, Hkv, T, 64, BF16, 64)
    k, v = (rnd(s, 2, Hkv, T, 64) for s in (1, 2))
    v[:, :, 3, 5], v[:, :, 70, 6], v[:, :, 71, 7] = math.inf, -math.inf, math.nan
    bd.cache_write(cache, k.to(DEV), v.to(DEV))
    counts = [n - 1, 0]
    got = attend(cache, rnd(3, 2, Hq, n, 64, dtype=BF16), [[T] * Hkv] * 2, counts, causal, T)
    assert (got[0, :, n - 1:] == 0).all() and (got[1] == 0).all()
    there = got[0, :, :n - 1]
    assert (there[..., 5] == math.inf).all() and (there[..., 6] == -math.inf).all()
    assert torch.isnan(there[..., 7]).all()
    assert torch.isfinite(there[..., :5]).all() and torch.isfinite(there[..., 8:]).all()


@pytest.mark.parametrize("Hq,n", [(2, 10), (2, 70)])
def test_queries_that_see_nothing_beside_infinite_values(Hq, n):
    """Fewer rows than queries: the first queries see none, also where the rows of the others hold infinities."""
    cache = make_cache(1, 1, 64, 64, BF16, 64)
    k, v = (rnd(s, 1, 1, 3, 64) for s in (1, 2))
    v[..., 0, 5], v[..., 0, 6] = math.inf, math.nan
    bd.cache_write(cache, k.to(DEV), v.to(DEV))
    got = attend(cache, rnd(3, 1, Hq, n, 64, dtype=BF16), [[3]])
    assert (got[:, :, :n - 3] == 0).all()
    assert (got[:, :, n - 3:, 5] == math.inf).all() and torch.isnan(got[:, :, n - 3:, 6]).all()
    assert torch.isfinite(got[:, :, n - 3:, 7:]).all()


@pytest.mark.parametrize("Hq,Hkv,T,n", SPLITS)
def test_a_nan_key_is_seen_through_splits(Hq, Hkv, T, n):
    """NaN in a key that the queries see, or in a query, makes their results NaN, however the keys are split,
    and leaves the other heads' as they are."""
    cache = make_cache(1, Hkv, T, 64, BF16, 64)
    k, v = (rnd(s, 1, Hkv, T, 64) for s in (1, 2))
    k[0, 1, 17, 9] = math.nan
    bd.cache_write(cache, k.to(DEV), v.to(DEV))
    q = rnd(3, 1, Hq, n, 64, dtype=BF16)
    q[0, 0, n - 1, 3] = math.nan
    got = attend(cache, q, [[T] * Hkv], causal=False, T=T)
    assert torch.isnan(got[:, Hq // 2:]).all() and torch.isnan(got[:, 0, n - 1]).all()
    assert torch.isfinite(got[:, 1:Hq // 2]).all() and torch.isfinite(got[:, 0, :n - 1]).all()


def close_bound(cache, q, lens):
    """(out, bound) in 64 bits without a causal limit, of an attention whose weights are rounded once and
    divided by the sum of what they were rounded to.  With p (1 + e), |e| <= u = 2^-8 (bf16), the quotient is
    off by sum p e (v - o) / sum p (1 + e), at most u / (1 - u) sum p |v - o| (p normalised): a rounding that
    all weights share falls out, and of one heavy weight what is left of it.  Beside it the result's own
    rounding, u |o|, and the fp32 terms of tests/paged.py, here `rel`, times sum p |v|."""
    q = q.double().numpy()
    B, Hq, n, d = q.shape
    Hkv = cache.k.shape[1]
    out, tol = np.zeros_like(q), np.zeros_like(q)
    for b in range(B):
        for c in range(Hkv):
            m = lens[b][c]
            k, v = paged.cached_rows(cache, b, c, m)
            for h in range(c * (Hq // Hkv), (c + 1) * (Hq // Hkv)):
                x = q[b, h] @ k.T / math.sqrt(d)
                size = np.abs(q[b, h]) @ np.abs(k).T / math.sqrt(d)
                p = np.exp(x - x.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                o = p @ v
                apart = np.stack([pi @ np.abs(v - oi) for pi, oi in zip(p, o)])
                rel = 2 * ((d + 4) * paged.U32 * size.max(1) + 2 * paged.U32) + 2 * m * paged.U32
                out[b, h] = o
                tol[b, h] = paged.U16 * np.abs(o) + paged.U16 / (1 - paged.U16) * apart \
                    + 1.01 * rel[:, None] * (p @ np.abs(v))
    return out, tol


@pytest.mark.parametrize("kind", [BF16, E4M3])
@pytest.mark.parametrize("B,Hq,Hkv,T,n", [(2, 28, 4, 321, 1), (8, 64, 32, 1111, 1), (8, 96, 32, 700, 10),
                                          (1, 8, 2, 3000, 5), (1, 8, 2, 321, 40),
                                          (1, 8, 2, 3000, 40)])
def test_weights_and_their_sum_are_rounded_alike(kind, B, Hq, Hkv, T, n):
    """Peaked rows (queries of standard deviation 4): the heaviest weight's rounding cancels in the quotient.
    (Not of int8 rows: their weights are rounded with the scale of V.)"""
    d = 128
    cache = make_cache(B, Hkv, T, d, kind, 64)
    k, v = (rnd(s, B, Hkv, T, d) for s in (1, 2))
    bd.cache_write(cache, k.to(DEV), v.to(DEV))
    q = (4 * rnd(3, B, Hq, n, d)).to(BF16)
    got = attend(cache, q, [[T] * Hkv] * B, causal=False, T=T).double().numpy()
    want, tol = close_bound(cache, q, [[T] * Hkv] * B)
    off = np.abs(got - want)
    print("relative 2-norm", np.linalg.norm(off) / np.linalg.norm(want), flush=True)
    assert (off <= tol).all(), (off / tol).max()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,Hq,Hkv,n", [(16, 16, 16, 1), (16, 64, 16, 8), (8, 64, 16, 40)])
def test_sums_of_large_values_stay_in_range(kind, B, Hq, Hkv, n):
    """Values of 2^116 under weights that grow once, after the first keys of every wave, by 2^3.7: sums relative
    to the largest weight are 2^10.3 times a value, which fp32 holds; relative to the first keys' weight they
    would be 2^13.9 times it, which fp32 does not."""
    T, d = 1500, 64
    cache = make_cache(B, Hkv, T, d, kind, 64)
    v = rnd(2, B, Hkv, 1, d).sign().expand(B, Hkv, T, d) * 2.0 ** 116
    k = torch.zeros(B, Hkv, T, d)
    k[:, :, 512:, 0] = 5.125
    bd.cache_write(cache, k.to(DEV), v.to(DEV))
    q = torch.zeros(B, Hq, n, d)
    q[..., 0] = 4.0
    check_attention(cache, q.to(BF16), [[T] * Hkv] * B, causal=False, T=T)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,T,n", SPLITS + [(4, 1, 77, 20)])
def test_e4m3_rows_of_any_scale(Hq, Hkv, T, n, d):
    """Scales that are no powers of two, as another program may have quantised its rows.  A value times its
    scale is rounded to bf16 where the staged kernel takes it: u |q| |k| more in a logit (p off by twice that,
    as in tests/paged.py), u sum p |v| more in the result; only in part of the rows' tiles."""
    cache = make_cache(1, Hkv, T, d, E4M3, 16)
    gen = torch.Generator().manual_seed(T + n)
    shape = tuple(cache.k.shape)
    for x, s, size in ((cache.k, cache.k_scale, 0.5), (cache.v, cache.v_scale, 3.0)):
        x.copy_((torch.randn(shape, generator=gen) * 16).to(E4M3).to(DEV))
        s.copy_((size / 16 * torch.exp2(2 * torch.rand(shape[:3], generator=gen) - 1)).to(DEV))
    s = cache.k_scale                              # a third of the pages as cache_write leaves them
    s[::3] = torch.exp2(torch.floor(torch.log2(s[::3])))
    q = (0.5 * rnd(3, 1, Hq, n, d)).to(BF16)
    lens = [[T] * Hkv]
    got = attend(cache, q, lens, T=T).double().numpy()
    want, tol = paged.attention(cache, q, torch.as_tensor(lens), None, True)
    for c in range(Hkv):
        k, v = paged.cached_rows(cache, 0, c, T)
        for h in range(c * (Hq // Hkv), (c + 1) * (Hq // Hkv)):
            size = np.abs(q[0, h].double().numpy()) @ np.abs(k).T / math.sqrt(d)
            x = q[0, h].double().numpy() @ k.T / math.sqrt(d)
            x = np.where(np.arange(T)[None] <= T - n + np.arange(n)[:, None], x, -np.inf)
            p = np.exp(x - x.max(1, keepdims=True))
            weight = (p / p.sum(1, keepdims=True)) @ np.abs(v)
            # (e^y - 1 <= y e^y)
            y = 2 * paged.U16 * size.max(1)[:, None]
            tol[0, h] += (paged.U16 + y * np.exp(y)) * 1.02 * weight
    off = np.abs(got - want)
    assert (off <= tol).all(), (off / tol).max()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("src", [F32, BF16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_written_infinities_and_nan(kind, src, d, bad):
    """No source row with an infinity or NaN reads back as numbers: bf16 keeps it in its place, e4m3 holds NaN
    there, an int8 row is NaN as a whole; rows beside it are as without it."""
    k, v = (rnd(s, 1, 2, 40, d).to(src) for s in (1, 2))
    k0, v0 = k.clone(), v.clone()
    at = [(0, 3, 5), (0, 17, d - 1), (1, 39, 0)]   # head, row, element
    for x in (k, v):
        for c, t, j in at:
            x[0, c, t, j] = bad
    lens = i32([[40, 40]])
    caches = [make_cache(1, 2, 40, d, kind, 16) for _ in range(2)]
    bd.cache_write(caches[0], k.to(DEV), v.to(DEV))
    bd.cache_write(caches[1], k0.to(DEV), v0.to(DEV))
    for got, want, x in zip(*(bd.cache_read(c, lens, 40, F32) for c in caches), (k, v)):
        got, want = got.cpu(), want.cpu()
        rows = torch.zeros(2, 40, dtype=torch.bool)
        for c, t, j in at:
            rows[c, t] = True
            if kind == I8:
                assert torch.isnan(got[0, c, t]).all()
            elif kind == E4M3:
                assert torch.isnan(got[0, c, t, j]) and torch.isnan(got[0, c, t]).sum() == 1
            else:
                assert torch.equal(got[0, c, t].nan_to_num(7e30), x[0, c, t].to(BF16).float().nan_to_num(7e30))
        assert torch.equal(got[0][~rows], want[0][~rows])
