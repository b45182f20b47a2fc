"""Plain 64-bit attention over a shared prefix (numpy; no code of the library), with the bounds of tests/paged.py."""
from __future__ import annotations

import math

import numpy as np

import paper_2607_22586_amd as mm
from paged import U16, U32, cached_rows


def attention(cache, q, lens, shared, shared_table, q_counts=None, causal=True):
    """(out, bound) [B, Hq, n, d]: rows below `shared` by shared_table, the others by the cache's table."""
    q = q.cpu().double().numpy()
    B, Hq, n, d = q.shape
    Hkv, G = cache.k.shape[1], shared.shape[0]
    gh, each, cap = Hq // Hkv, B // G, cache.table.shape[1] * cache.k.shape[2]
    prefix = mm.PagedCache(cache.k, cache.v, cache.k_scale, cache.v_scale, shared_table)
    lens, shared = lens.cpu().numpy(), shared.cpu().numpy()
    out, tol = np.zeros_like(q), np.zeros_like(q)
    for b in range(B):
        nq = n if q_counts is None else int(min(max(int(q_counts[b]), 0), n))
        for c in range(Hkv):
            m = int(min(max(int(lens[b, c]), 0), cap))
            s = int(min(max(int(shared[b // each, c]), 0), m))
            if m == 0 or nq == 0:
                continue
            k, v = (np.concatenate([x, y[s:]]) for x, y in zip(cached_rows(prefix, b // each, c, s),
                                                               cached_rows(cache, b, c, m)))
            for h in range(c * gh, (c + 1) * gh):
                x = q[b, h, :nq] @ k.T / math.sqrt(d)
                size = np.abs(q[b, h, :nq]) @ np.abs(k).T / math.sqrt(d)
                seen = np.ones_like(x, bool)
                if causal:
                    seen = np.arange(m)[None] <= m - nq + np.arange(nq)[:, None]
                any_ = seen.any(1)
                x = np.where(seen, x, -np.inf)
                p = np.exp(x - np.where(any_, x.max(1), 0.0)[:, None])
                p /= np.where(any_, p.sum(1), 1.0)[:, None]
                out[b, h, :nq] = p @ v
                rel = 2 * ((d + 4) * U32 * np.where(seen, size, 0).max(1) + 2 * U32) + 2 * m * U32
                tol[b, h, :nq] = U16 * np.abs(out[b, h, :nq]) + (U16 + rel[:, None]) * (p @ np.abs(v))
    return out, tol
