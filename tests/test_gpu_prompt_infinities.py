"""Prompt attention with infinities in k, against the 64-bit form without the keys that they take out."""
import math

import numpy as np
import pytest

import paper_2607_22586_amd as mm
from paged import U16, U32
from test_gpu_prompt import inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("T", [70, 400])
def test_infinities_in_k(d, causal, T):
    """A logit of -inf takes the key's weight and no more; one of +inf, or of 0 times an infinity, makes the row and its
    log-sum-exp NaN."""
    q, k, v = inputs(1, 4, 2, T, d, 17)
    at, dim = 33, 5
    k[:, :, at, dim] = float("inf")
    q[:, 3, ::7, dim] = 0.0
    out, lse = mm.prompt_attention(q, k, v, causal=causal, with_lse=True)
    out, lse = out.cpu().double().numpy()[0], lse.cpu().double().numpy()[0]
    q, k, v = (x[0].cpu().double().numpy() for x in (q, k, v))
    k[:, at, dim] = 0.0
    for h in range(4):
        seen = np.tril(np.ones((T, T), bool)) if causal else np.ones((T, T), bool)
        sees = seen[:, at].copy()
        lost = sees & (q[h, :, dim] >= 0)
        assert np.isnan(out[h, lost]).all() and np.isnan(lse[h, lost]).all() and lost.any()
        seen[:, at] = ~sees & seen[:, at]
        kk, vv = k[h // 2], v[h // 2]
        x = np.where(seen, q[h] @ kk.T / math.sqrt(d), -np.inf)
        size = np.where(seen, np.abs(q[h]) @ np.abs(kk).T / math.sqrt(d), 0).max(1)
        here = ~lost
        most = x[here].max(1)
        p = np.exp(x[here] - most[:, None])
        total = p.sum(1)
        p /= total[:, None]
        want, rel = p @ vv, (2 * ((d + 4) * U32 * size[here] + 2 * U32) + 2 * T * U32)[:, None]
        assert (np.abs(out[h, here] - want) <= U16 * np.abs(want) + (U16 + rel) * (p @ np.abs(vv))).all()
        assert (np.abs(lse[h, here] - most - np.log(total)) <= rel[:, 0] + 4 * U32 * (size[here] + 40)).all()
