"""Plain 64-bit forms of the paged-cache operators for the tests (numpy and CPU
torch; no code of the library), and the bounds of their comparison.

Bounds.  Half a step of a type is u = finfo(t).eps / 2 relative to the value
(bf16 2^-8, fp32 2^-24).  An output o = sum p_t v_t / sum p_t of the attention
is off by
  * its own rounding to bf16: u_bf16 |o|;
  * each p's rounding to bf16 for the product with v: u_bf16 sum p_t |v_t| (p
    normalised);
  * the logits: products of bf16 values are exact in fp32 and d of them are
    added, so a logit x = q . k / sqrt(d) is off by at most (d + 4) u_fp32 S,
    S = sum |q_j k_j| / sqrt(d) (4: its scale, the two scales of an 8-bit row
    and the subtraction of the maximum, each once; the maximum itself is a
    logit, at most max S large, and its subtraction is counted with max S).
    A factor of 2^x is off relatively by that much, plus 2 u_fp32 of the
    exponential, numerator and denominator both;
  * fp32 sums over T rows, numerator and denominator: 2 T u_fp32.
All of them multiply sum p_t |v_t|.
"""
from __future__ import annotations

import math

import numpy as np
import torch

U16, U32 = 2.0 ** -8, 2.0 ** -24

# the 256 e4m3 values: 4 exponent bits (bias 7), 3 mantissa bits, no infinities
_CODES = np.arange(256)
_E, _M = (_CODES >> 3) & 15, _CODES & 7
E4M3 = np.where(_E == 0, _M * 2.0 ** -9, (1 + _M / 8) * 2.0 ** (_E - 7.0)) * np.where(_CODES >> 7, -1.0, 1.0)
E4M3[[127, 255]] = np.nan


def e4m3_codes(y):
    """Codes of the e4m3 values nearest to y (|y| <= 448), ties to the even code, zeros positive."""
    mag = E4M3[:127]
    a = np.abs(y)
    hi = np.clip(np.searchsorted(mag, a), 1, 126)
    lo = hi - 1
    up = (mag[hi] - a < a - mag[lo]) | ((mag[hi] - a == a - mag[lo]) & (hi % 2 == 0))
    code = np.where(up, hi, lo)
    return np.where((y < 0) & (code > 0), code + 128, code)


def quantised(x, kind):
    """Rows x [..., d] (fp32 array) as the cache holds them: (values in 64 bits without their scale, scales)."""
    x = np.asarray(x, np.float32)
    if kind == torch.bfloat16:
        return torch.from_numpy(x.copy()).to(torch.bfloat16).double().numpy(), None
    a = np.abs(x).max(-1, keepdims=True)
    if kind == torch.float8_e4m3fn:
        f, e = np.frexp(a.astype(np.float64))      # a = f 2^e, 448 = 0.875 * 2^9
        s = np.ldexp(1.0, np.maximum(e - 9 + (f > 0.875), -126))
        s = np.where(a > 0, s, 2.0 ** -126)
        return E4M3[e4m3_codes(x.astype(np.float64) / s)], s[..., 0]
    a = np.maximum(a, np.float32(2.0 ** -100))
    y = np.rint(x * (np.float32(127) / a))
    return y.astype(np.float64), (a / np.float32(127))[..., 0].astype(np.float64)


def held(pages):
    """A pool's values in 64 bits (e4m3 and int8 without their scales), on the CPU."""
    if pages.dtype == torch.float8_e4m3fn:
        return E4M3[pages.cpu().view(torch.uint8).numpy()]
    return pages.cpu().double().numpy()


def cached_rows(cache, b, c, n):
    """(K, V) [n, d] in 64 bits: the first n cached rows of (b, c); zero rows of pages outside the pool."""
    page = cache.k.shape[2]
    table = cache.table.cpu().numpy()
    got = []
    for pages, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        x = np.zeros((n, pages.shape[3]))
        for j in range(-(-n // page)):
            p = int(table[b, j])
            if not 0 <= p < pages.shape[0]:
                continue
            rows = held(pages[p, c])
            if scale is not None:
                rows = rows * scale[p, c].cpu().double().numpy()[:, None]
            x[j * page:(j + 1) * page] = rows[:n - j * page]
        got.append(x)
    return got


def attention(cache, q, lens, q_counts=None, causal=True):
    """(out, bound) [B, Hq, n, d] in 64 bits: the attention of chunk queries, and how far a result may be off."""
    q = q.cpu().double().numpy()
    B, Hq, n, d = q.shape
    Hkv = cache.k.shape[1]
    lens = lens.cpu().numpy()
    out, tol = np.zeros_like(q), np.zeros_like(q)
    cap = cache.table.shape[1] * cache.k.shape[2]
    for b in range(B):
        nq = n if q_counts is None else int(min(max(int(q_counts[b]), 0), n))
        for c in range(Hkv):
            m = int(min(max(int(lens[b, c]), 0), cap))
            if m == 0 or nq == 0:
                continue
            k, v = cached_rows(cache, b, c, m)
            for h in range(c * (Hq // Hkv), (c + 1) * (Hq // Hkv)):
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
