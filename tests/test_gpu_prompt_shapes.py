"""Prompt attention in each of its launch shapes: row tiles that two workgroups have, long packed sequences, and every
key by a query that has all its weight there."""
import math

import pytest
import torch

import paper_2607_22586_amd as mm
from paged import U16, U32
from test_gpu_prompt import DEV, check, inputs, int32

pytestmark = pytest.mark.gpu

# (d, Hq, Hkv, T): as the launch has its workgroups, of four and eight waves, with one, two and four groups of keys
FEW, TWO, ONE = (64, 4, 4, 1500), (64, 7, 7, 4100), (64, 16, 16, 4100)


@pytest.mark.parametrize("shape,cuts", [
    (FEW, [0, 100, 1500]),                         # a short sequence before a long one
    (FEW, [0, 700, 1500]),                         # two long ones
    (FEW, [0, 1400, 1500]),
    ((128, 7, 1, 1500), [2, 60, 1499]),
    ((128, 2, 2, 2600), [0, 1000, 1000, 1030, 2590]),
    (TWO, [0, 1000, 1001, 1001, 1040, 2900, 4100]),
    (TWO, [0, 40, 70, 71, 4000, 4000, 4090]),
    (ONE, [0, 1000, 1001, 1001, 1040, 2900, 2950, 4100]),
    (ONE, [3, 30, 31, 1500, 1530, 1550, 4095]),
    (ONE, [0, 0, 2000, 2100, 2100, 4100])])
def test_row_tiles_of_several_long_sequences(shape, cuts):
    d, Hq, Hkv, T = shape
    assert T // (len(cuts) - 1) >= 512
    q, k, v = inputs(1, Hq, Hkv, T, d, len(cuts), "tokens")
    out = torch.full_like(q, 7.0)
    lse = torch.full((1, Hq, T), 7.0, device=DEV)
    mm.prompt_attention(q, k, v, starts=int32(cuts), causal=False, out=out, lse=lse)
    check(out, q, k, v, cuts, False, lse)
    for x in (out, lse):
        assert bool((x[:, :, :cuts[0]] == 7.0).all()) and bool((x[:, :, cuts[-1]:] == 7.0).all())
    again = torch.full_like(q, 7.0)
    mm.prompt_attention(q, k, v, starts=int32(cuts), causal=False, out=again)
    assert torch.equal(again, out)


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 9, 9), (64, 9, 9), (128, 10, 2)])
@pytest.mark.parametrize("causal", [True, False])
def test_long_packed_sequences(d, Hq, Hkv, causal):
    """Two sequences of more than 8192 tokens against the formula in fp32, with test_as_in_fp32's bound."""
    T, cuts = 16420, [3, 8300, 16411]
    q, k, v = inputs(1, Hq, Hkv, T, d, Hq, "tokens")
    out = torch.full_like(q, 7.0)
    lse = torch.full((1, Hq, T), 7.0, device=DEV)
    mm.prompt_attention(q, k, v, starts=int32(cuts), causal=causal, out=out, lse=lse)
    for x in (out, lse):
        assert bool((x[:, :, :cuts[0]] == 7.0).all()) and bool((x[:, :, cuts[-1]:] == 7.0).all())
    for h in range(Hq):
        for lo, hi in zip(cuts, cuts[1:]):
            n, c = hi - lo, h // (Hq // Hkv)
            qq, kk, vv = q[0, h, lo:hi].float(), k[0, c, lo:hi].float(), v[0, c, lo:hi].float()
            x = qq @ kk.t().contiguous() * d ** -0.5
            size = float((qq.abs() @ kk.abs().t().contiguous()).max()) * d ** -0.5
            if causal:
                t = torch.arange(n, device=DEV)
                x = x.masked_fill(t > t[:, None], -float("inf"))
            p = torch.softmax(x, -1)
            want = p @ vv
            rel = 4 * ((d + 4) * U32 * size + 2 * U32) + 4 * n * U32
            assert bool(((out[0, h, lo:hi].float() - want).abs() <= U16 * want.abs() + (U16 + rel) * (p @ vv.abs())).all())
            assert float((lse[0, h, lo:hi] - torch.logsumexp(x, -1)).abs().max()) <= rel + 4 * U32 * (size + 40)


@pytest.mark.parametrize("d,Hq,Hkv,T,cuts", [
    (64, 2, 2, 5000, None), (64, 2, 2, 40, None), (64, 15, 15, 1300, None), (64, 30, 2, 1300, None),
    (64, 9, 9, 8300, None), (64, 40, 40, 1300, [0, 400, 800, 1300]), (64, 8, 8, 1500, [0, 400, 800, 1300, 1500]), (64, 4, 2, 2500, [0, 100, 1300, 2490]),
    (64, 4, 4, 1500, list(range(0, 1501, 60))), (128, 2, 1, 3000, None), (128, 9, 9, 8300, None),
    (128, 3, 1, 3000, [0, 700, 701, 2900, 3000]), (128, 7, 1, 900, list(range(0, 901, 75)))])
@pytest.mark.parametrize("causal", [True, False])
def test_key_by_key(d, Hq, Hkv, T, cuts, causal):
    """Nearly all of a query's weight on one key: its own, then another that it sees, so that each key has a query.

    Key t is its 14 bits as -1 and 1, the query f times those of its key (f = 128 at d = 64, 192 at 128), so that
    a key j bits away has at most e^(-32 j) times the weight: together less than 14 e^-32 1.001 < 1.8e-13, of
    values at most 12 away: 2.2e-12, beside the rounding of the result.  The key's logit, x = 14 f / sqrt(d), is
    exact up to the scale's and one product's rounding, and the log-sum-exp is x + ln(1 + 1.8e-13): its own
    steps (the difference to the reference, the exponential, the logarithm, the sum, the product with ln 2) are off by
    less than 8 u_fp32 (x + 16), where a key left out or counted twice would be off by ln 2 or more."""
    f, bits = (128 if d == 64 else 192), 14
    at = torch.arange(T, device=DEV)
    code = ((at[:, None] >> torch.arange(bits, device=DEV)) & 1) * 2.0 - 1
    k = torch.zeros((1, Hkv, T, d), device=DEV)
    k[..., :bits] = code
    g = torch.Generator(device=DEV)
    g.manual_seed(T)
    v = torch.randn((1, Hkv, T, d), generator=g, device=DEV).clamp(-6, 6).bfloat16()
    lo, hi = torch.zeros_like(at), torch.full_like(at, T)
    if cuts:
        edges = torch.tensor(cuts, device=DEV)
        lo = edges[torch.searchsorted(edges, at, right=True) - 1]
        hi = edges[torch.searchsorted(edges, at, right=True).clamp(max=len(cuts) - 1)]
    inside = (at >= cuts[0]) & (at < cuts[-1]) if cuts else torch.ones_like(at, dtype=torch.bool)
    if causal:
        hi = at + 1
    x = bits * f / math.sqrt(d)
    starts = None if cuts is None else int32(cuts)
    other = torch.stack([lo + (torch.rand(T, generator=g, device=DEV) * (hi - lo)).long().minimum(hi - lo - 1).clamp(min=0) for _ in range(Hq)])
    if not causal:                                 # (a turn of the sequence: every key is some query's)
        other = lo + (at - lo + torch.arange(1, Hq + 1, device=DEV)[:, None] * 37) % (hi - lo).clamp(min=1)
    for key in (at.expand(Hq, -1), other.clamp(max=T - 1)):
        q = torch.zeros((1, Hq, T, d), device=DEV)
        q[0, ..., :bits] = f * code[key]
        out, lse = mm.prompt_attention(q.bfloat16(), k.bfloat16(), v, starts=starts, causal=causal, with_lse=True)
        head = torch.arange(Hq, device=DEV)[:, None] // (Hq // Hkv)
        want = v[0, head, key].double()
        off = (out[0].double() - want).abs()
        assert bool((off <= U16 * want.abs() + 2.2e-12)[:, inside].all())
        assert float((lse[0].double() - x).abs()[:, inside].max()) <= 8 * U32 * (x + 16)
