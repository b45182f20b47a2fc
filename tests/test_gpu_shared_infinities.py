"""Infinities and NaN in shared rows reach the sequences that see them, and no others of their group."""
import pytest
import torch

import paper_2607_22586_amd as mm
from shared import attention
from test_gpu_shared import DEV, TYPES, int32, problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,d,n", [(1, 1, 64, 1), (7, 1, 128, 1), (32, 2, 64, 1), (16, 2, 128, 3), (80, 2, 64, 2),
                                        (28, 4, 128, 9)])
@pytest.mark.parametrize("causal", [True, False])
def test_sequences_that_do_not_see_the_row(dtype, Hq, Hkv, d, n, causal):
    """Rows 150 of V and 180 of K of a prompt of 200: sequences of fewer rows are as without them, bit for bit."""
    B, G = 8, 2
    cache, q, lens, shared, table = problem(B, G, Hq, Hkv, d, dtype, 32, 200, 40, n, 9, poison=False)
    lens = int32([[x] * Hkv for x in (240, 150, 0, 201, 97, 200, 230, 31)])
    shared = int32([[200] * Hkv, [190] * Hkv])
    want = mm.shared_attention(q, cache, lens, shared, table, causal=causal)
    out, tol = attention(cache, q, lens, shared, table, causal=causal)
    assert bool((abs(want.cpu().double().numpy() - out) <= tol).all())
    for x in (float("nan"), float("inf"))[:2 if dtype == torch.bfloat16 else 1]:
        for g in range(G):
            for rows, scale, t in ((cache.v, cache.v_scale, 150), (cache.k, cache.k_scale, 180)):
                page, slot = int(table[g, t // 32]), t % 32
                if dtype == torch.bfloat16:
                    rows[page, :, slot, 5] = x
                elif dtype == torch.float8_e4m3fn:
                    rows.view(torch.uint8)[page, :, slot, 5] = 0x7F
                else:
                    scale[page, :, slot] = x
        got = mm.shared_attention(q, cache, lens, shared, table, causal=causal)
        few = [b for b in range(B) if int(lens[b, 0]) <= 150]
        assert len(few) == 4
        assert torch.equal(got[few], want[few])
        for b in set(range(B)) - set(few):         # (the last query of each sees all its rows)
            assert bool((~got[b, :, -1].isfinite()).any(-1).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,Hq,T,n", [(40, 4, 3000, 1), (6, 12, 700, 9), (3, 2, 5000, 1)])
def test_most_sequences_have_fewer_rows(dtype, B, Hq, T, n):
    """Lengths anywhere below the shared rows, against the 64-bit form: nothing of other sequences' rows or logits is
    left in their sums, however large."""
    cache, q, lens, shared, table = problem(B, 1, Hq, 1, 64, dtype, 64, T, 20, n, 3, poison=False)
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, T, (B, 1), generator=g).int()
    lens[0], lens[-1] = T + 7, T
    lens, shared = lens.to(DEV), int32([[T]])
    q[1::2] *= 12                                  # (logits to hundreds)
    for causal in (True, False):
        got = mm.shared_attention(q, cache, lens, shared, table, causal=causal)
        out, tol = attention(cache, q, lens, shared, table, causal=causal)
        assert bool((abs(got.cpu().double().numpy() - out) <= tol).all())
