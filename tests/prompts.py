"""Plain 64-bit attention of prompts over themselves (CPU; no code of the library), with the bounds of tests/paged.py.

The log-sum-exp: the logits' error, (d + 4) u_fp32 S with S = sum |q_j k_j| / sqrt(d), and that of the reference m,
which is subtracted before and added after (counted with max S once more); the sum of T weights, T u_fp32 and 2 u_fp32
of each exponential, relative and so absolute in the logarithm; the logarithm (2 u_fp32 of |log l|, which is at most
16 ln 2 + ln T here, the reference being up to 2^8 above the largest weight) and the roundings of m + log2 l and of its product with ln 2 (with ln 2's
own: 3 u_fp32 |lse|, and u_fp32 |m|)."""
from __future__ import annotations

import math

import numpy as np

from paged import U16, U32


def spans(starts, T):
    if starts is None:
        return [(0, T)]
    at = [min(max(int(x), 0), T) for x in starts]
    return [(a, b) for a, b in zip(at, at[1:]) if a < b]


def attention(q, k, v, starts=None, causal=True):
    """(out, out's bound, lse, lse's bound) in 64 bits; NaN in rows of no sequence."""
    q, k, v = (x.cpu().double().numpy() for x in (q, k, v))
    B, Hq, T, d = q.shape
    gh = Hq // k.shape[1]
    out, tol = np.full_like(q, np.nan), np.zeros_like(q)
    lse, ltol = np.full(q.shape[:3], np.nan), np.zeros(q.shape[:3])
    for b in range(B):
        for h in range(Hq):
            for lo, hi in spans(starts, T):
                n, c = hi - lo, h // gh
                kk, vv = k[b, c, lo:hi], v[b, c, lo:hi]
                x = q[b, h, lo:hi] @ kk.T / math.sqrt(d)
                size = np.abs(q[b, h, lo:hi]) @ np.abs(kk).T / math.sqrt(d)
                seen = np.tril(np.ones((n, n), bool)) if causal else np.ones((n, n), bool)
                x = np.where(seen, x, -np.inf)
                most = x.max(1)
                p = np.exp(x - most[:, None])
                total = p.sum(1)
                p /= total[:, None]
                out[b, h, lo:hi] = p @ vv
                lse[b, h, lo:hi] = most + np.log(total)
                big = np.where(seen, size, 0).max(1)
                logits = (d + 4) * U32 * big
                rel = 2 * (logits + 2 * U32) + 2 * n * U32
                tol[b, h, lo:hi] = U16 * np.abs(out[b, h, lo:hi]) + (U16 + rel[:, None]) * (p @ np.abs(vv))
                ltol[b, h, lo:hi] = 2 * logits + (n + 2) * U32 + 2 * U32 * (16 * math.log(2) + math.log(n)) \
                    + 4 * U32 * (np.abs(lse[b, h, lo:hi]) + 16)
    return out, tol, lse, ltol
